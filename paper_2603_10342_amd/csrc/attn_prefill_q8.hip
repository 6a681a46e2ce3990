// Cold and resume prefill over the 8-bit paged KV cache, bf16: causal attention of ragged chunks behind cached prefixes, any group
// size, head_dim a multiple of 16 up to 256.
//
// A dense contraction, bound by the matrix cores.  A workgroup of NW waves owns 32 * NW columns of one (session, KV head), a
// column being a (token, query head of the group) pair; a wave owns 32 of them with their queries in registers, and takes keys and
// values 64 at a time in the tile arithmetic of the bf16 caches (attn_tile32.h).  What differs is how a tile comes into LDS:
// its bytes go through registers, one tile ahead, and are written as bf16 numbers, their powers of two multiplied in (exactly).
// Done once a workgroup that is an eighth (NW = 8) of what a conversion behind LDS would cost each wave, and the products run as
// they do over a bf16 cache.  A wave brings one 16-token group of the tile (or half of one): one page id, 16 exponent bytes.
//   iteration t: K(t + 2) and V(t + 1) requested into registers; S(t) = K(t) Q^T, and between its products K(t + 1) and V(t), which are
//   in registers, converted and written to LDS; P(t) side by side with O += V(t - 1) P(t - 1); barrier.
// The conversions - 40 vector instructions a wave and tile at NW = 8 and 128 channels, beside 100 of the softmax - so run while the vector units
// have nothing else; ahead of the products eight prompts of 4096 tokens took 1222 us, so 1134 (970 TFLOP/s).  Over a bf16 cache,
// whose tiles need no conversion, they take 1026 where these take 1100 (one session of measurements); 8 of 512 38.6 and 45.1, one of 2048 51 and 57, 32 chunks of
// 128..1024 rows on 2048..8192 tokens 1770 and 1812.
// Weights are rounded to bf16 for the value product at every shape, where bf16 caches have that for 128 channels on pages of 16 only: an error of up to
// 2^-8 of a weight, each for itself, beside 2^-4 of a cached value and 2^-8 of the output.  As three terms, 24 bits: eight prompts of 2000 x 64 202 -> 307 us,
// x 256 776 -> 1229, eight of 4096 x 128 1124 -> 2129 (by attn_split_q8.hip: tiles spill); 64-bit attention over the cached numbers differs from the output by 1.05 to 1.33 times
// what the output's own rounding leaves.  fp32 activations, which keep 24 bits, and few rows take attn_split_q8.hip (split_preferred()).
#include <algorithm>
#include <atomic>

#include "attn_tile32.h"
#include "q8_internal.h"
#include "tile_list.h"

namespace ag {
namespace q8 {
namespace {

using tile32::BN;
using tile32::Weights;
using tile32::f32x16;
using tile32::tile_bytes;

// two key and two value tiles
constexpr int lds_bytes(int dt) { return 4 * tile_bytes(dt); }

template <int NW, int DT, bool kExact>
__global__ __launch_bounds__(64 * NW, DT > 128 ? 1 : 2) void prefill_q8_kernel(Args x, Deal deal)
{
    constexpr int kCols = 32 * NW, kTile = tile_bytes(DT);
    constexpr int kWavesPerGroup = NW / 4, kPer = DT / 64 / kWavesPerGroup;       // 16-byte pieces of a lane for a K tile, and for a V tile
    static_assert(kPer >= 1, "a wave brings whole pieces");
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];           // [2 K tiles][2 V tiles]

    const AttnArgs& a = x.a;
    const int hkv = a.c.hkv, hq = a.hq, G = hq / hkv, D = kExact ? DT : a.c.d, ps = a.c.ps, chunks = D >> 4;
    int g, j;
    if (!place_of(deal, hkv, g, j)) return;
    int s = -1, qt = 0, N = 0, P = 0, row0 = 0;
    find_tile<kCols>(a, j, G, s, qt, N, P, row0);
    if (s < 0) return;                              // beyond the batch's tiles
    const int ctx = P + N;
    const int col0 = qt * kCols, cols = min(N * G - col0, kCols);             // valid columns of the workgroup
    const Columns columns(col0, G);
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hi = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cols_w = max(0, min(32, cols - 32 * w));
    const int n_tiles = (P + columns.token(cols - 1)) / BN + 1;               // tiles the workgroup stages
    const int wave_tiles = cols_w > 0 ? (P + columns.token(32 * w + cols_w - 1)) / BN + 1 : 0;      // tiles this wave uses
    const int first_masked = (P + columns.token(32 * w) + 1) / BN;            // first tile holding a key this wave's first column may not see
    const int diagonal = n_tiles - (P + columns.token(0) + 1) / BN;           // how many of the last may hold a key that some column does not see
    const int col = min(32 * w + n, cols - 1);                                // columns beyond the tile repeat the last one
    const int token = columns.token(col), head = columns.head(col, token);
    const int qpos = P + token;
    const int64_t row = ((int64_t)row0 + token) * hq + (int64_t)g * G + head;

    // ---- tile requests: this wave's group of the tile, 16 keys; pieces [chunk][key] of the keys, [channel] of the values ----
    const int last_grp = (ctx - 1) >> 4, gshift = a.c.ps_shift - 4, gmask = (1 << gshift) - 1;
    const Finder find(a.c, D, g);
    const int my_grp = w / kWavesPerGroup, piece0 = (w % kWavesPerGroup) * kPer * 64 + lane;
    const int key = lane & 15;                                                // of the group, in every piece of a lane
    // Page ids of 64 groups, 16 tiles, a lane each, and of the next 64: everything that is in flight in the loop is a vector load, as a
    // scalar one shares its counter with the LDS operands and turns every wait for one of them into a wait for all.
    auto ids_of = [&](int win) { return a.bt[(int64_t)s * a.max_pages + (min(win * 64 + lane, last_grp) >> gshift)]; };
    int ids = ids_of(0), next_ids = ids_of(1);
    struct Raw { u32x4 k[kPer], v[kPer]; uint32_t ke, ve; };                  // ke: this lane's key's byte; ve: word lane & 3 of the values' 16
    // (uniform bases and 32-bit offsets of the lanes, the same for every tile: four 64-bit addresses kept in registers made the loop spill)
    const uint32_t k_off = (uint32_t)((key >> 2) * chunks * 64 + (key & 3) * 16 + (piece0 >> 4) * 64), v_off = (uint32_t)(piece0 * 16);
    const uint32_t ke_off = (uint32_t)key_place(key), ve_off = (uint32_t)(ps + (lane & 3) * 4);
    auto request_k = [&](int t, int page, Raw& x8) {
        const Where w8 = find.at(page, min(t * 4 + my_grp, last_grp) & gmask);
        const uint8_t* kp = data_at(a.c.k, w8.data);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            x8.k[i] = u32x4{0, 0, 0, 0};
            if (kExact || (piece0 >> 4) + i * 4 < chunks) x8.k[i] = *reinterpret_cast<const u32x4*>(kp + (k_off + i * 256));
        }
        x8.ke = exps_at(x.exps, w8.exps)[ke_off];
    };
    auto request_v = [&](int t, int page, Raw& x8) {
        const Where w8 = find.at(page, min(t * 4 + my_grp, last_grp) & gmask);
        const uint8_t* vp = data_at(a.c.v, w8.data);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            x8.v[i] = u32x4{0, 0, 0, 0};
            if (kExact || piece0 + i * 64 < D) x8.v[i] = *reinterpret_cast<const u32x4*>(vp + (v_off + i * 1024));
        }
        x8.ve = *reinterpret_cast<const uint32_t*>(exps_at(x.exps, w8.exps) + ve_off);
    };
    // Into LDS as bf16: K [chunk of 8 channels][64 keys], V [chunk of 8 keys][channel], 16-byte pieces, in kUnits steps of about four
    // instructions: of every piece the two halves of its keys, then the eight pairs of its values.
    constexpr int kUnits = 10 * kPer;
    unsigned char* const k_put = lds + (my_grp * 16 + key) * 16;
    unsigned char* const v_put = lds + 2 * kTile + my_grp * (DT * 32);
    struct Put { float e[16]; u32x4 y; };                                     // the values' powers, a piece in the making
    bool noted = false;                                                      // NaN among the values that this wave brought in
    auto begin_put = [&](int t, Raw& x8, Put& p) {
        const int keep = ctx - (t * BN + my_grp * 16);
        if (t + diagonal >= n_tiles) {                      // uniform
            asm volatile("");                                // (a branch, not a select for every word)
            if (keep < 16) {                                 // slots behind the last token may hold anything, NaN included: zeros
                asm volatile("");
                x8.ve = keep_bytes(x8.ve, keep - 4 * (lane & 3));        // (a byte of zero is a power of zero: a stale one may be an infinity)
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) x8.v[i][k] = keep_bytes(x8.v[i][k], keep - 4 * k);
            }
            noted |= take_nan_out(x8.v);                     // (nan_to_those_that_see_it())
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) p.e[i] = power(((uint32_t)__builtin_amdgcn_readlane((int)x8.ve, i >> 2) >> (8 * (i & 3))) & 0xFFu);
    };
    auto put_unit = [&](int unit, int t, const Raw& x8, Put& p) {             // keys of tile t + 1, values of tile t
        const int i = unit / 10, u = unit % 10;
        if (u < 2) {
            const int chunk = (piece0 + i * 64) >> 4;
            *reinterpret_cast<bf16x8*>(k_put + ((t + 1) & 1) * kTile + chunk * 2048 + u * 1024) = widen8(x8.k[i][2 * u], x8.k[i][2 * u + 1], power(x8.ke));
        } else {                                             // half: slots half * 4 + {0..3} and 8 + half * 4 + {0..3}
            const int half = (u - 2) >> 2, pair = (u - 2) & 3, word = half + (pair & 2), o = word * 4 + (pair & 1) * 2;
            p.y[pair] = pair & 1 ? widen_pair<true>(x8.v[i][word], p.e[o], p.e[o + 1]) : widen_pair<false>(x8.v[i][word], p.e[o], p.e[o + 1]);
            if (pair == 3) *reinterpret_cast<u32x4*>(v_put + (t & 1) * kTile + half * (DT * 16) + (piece0 + i * 64) * 16) = p.y;
        }
    };

    Raw ra, rb;
    request_k(0, __builtin_amdgcn_readlane(ids, my_grp), rb);

    // ---- Q^T as B operand: column n, k-step ks covers channels ks * 16 + hi * 8 .. + 7 ----
    bf16x8 qf[DT / 16];
    {
        const __bf16* qp = (const __bf16*)a.q + row * D + hi * 8;
#pragma unroll
        for (int ks = 0; ks < DT / 16; ++ks) {
            qf[ks] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (kExact || ks < chunks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
        }
    }
    const float sl2 = a.scale * tile32::kLog2e;
    float m = -INFINITY, lsum = 0.f;
    f32x16 o[DT / 32];
#pragma unroll
    for (int mb = 0; mb < DT / 32; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[mb][i] = 0.f;

    // what iteration 0 finds: K(0) in LDS, K(1) and V(0) on their way; tile t's page is that of K(t) now and of V(t) an iteration later
    int page = __builtin_amdgcn_readlane(ids, my_grp);
    request_v(0, page, ra);
    page = __builtin_amdgcn_readlane(ids, min(4, 4 * (n_tiles - 1)) + my_grp);
    request_k(min(1, n_tiles - 1), page, ra);
    {
        Put none;
#pragma unroll
        for (int unit = 0; unit < kUnits; ++unit)
            if (unit % 10 < 2) put_unit(unit, -1, rb, none);
    }
    __syncthreads();

    const unsigned char* const k_lane = lds + n * 16 + hi * 1024;
    const unsigned char* const v_lane = lds + 2 * kTile + n * 16 + hi * (DT * 16);
    Weights<false> pa, pb;
    // Requests past the last tile repeat it; what they bring is written to a place that nobody reads.
    auto iter = [&](int t, Weights<false>& p_prev, Weights<false>& p_cur, Raw& now, Raw& next) {
        const int tk = min(t + 2, n_tiles - 1);
        request_v(min(t + 1, n_tiles - 1), page, next);
        if (((t + 2) & 15) == 0) {                                            // K(t + 2) is the next window's first
            ids = next_ids;
            next_ids = ids_of(((t + 2) >> 4) + 1);
        }
        if (t + 2 < n_tiles) page = __builtin_amdgcn_readlane(ids, (tk & 15) * 4 + my_grp);
        request_k(tk, page, next);
        const bool do_sm = t < wave_tiles, do_pv = t >= 1 && t - 1 < wave_tiles;
        const unsigned char* kb = k_lane + (t & 1) * kTile;
        const unsigned char* vb = v_lane + ((t + 1) & 1) * kTile;             // V(t - 1)
        Put put;
        f32x16 sc[2];
        begin_put(t, now, put);
        if (do_sm) {
            constexpr int kSteps = DT / 8;
            tile32::qk_tile<DT>(kb, qf, sc, [&](int i) {
#pragma unroll
                for (int unit = i * kUnits / kSteps; unit < (i + 1) * kUnits / kSteps; ++unit) put_unit(unit, t, now, put);
            });
            if (t >= first_masked) {                                          // the tile straddles this wave's diagonal
                const int kbase = t * BN + hi * 4;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int at = kbase + b * 32 + (i >> 2) * 8 + (i & 3);
                        sc[b][i] = at <= qpos ? sc[b][i] : -INFINITY;
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) asm volatile("" : "+v"(now.k[i]), "+v"(now.v[i]));      // (else this is done ahead of the branch, for both sides)
#pragma unroll
            for (int unit = 0; unit < kUnits; ++unit) put_unit(unit, t, now, put);
        }
        tile32::softmax_and_value_product<DT, false>(do_sm, do_pv, vb, sc, sl2, m, lsum, p_prev, p_cur, o);
        __syncthreads();
    };
#pragma unroll 1
    for (int t = 0; t <= n_tiles; t += 2) {
        iter(t, pb, pa, ra, rb);
        if (t + 1 <= n_tiles) iter(t + 1, pa, pb, rb, ra);
    }

    uint32_t* const s_noted = reinterpret_cast<uint32_t*>(lds);               // (the tiles are done with)
    if (lane == 0) s_noted[w] = noted;
    __syncthreads();
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) any |= s_noted[i];
    if (any != 0 && cols_w > 0) nan_to_those_that_see_it<DT / 32>(a, find, s, (n_tiles - diagonal) * BN, P + columns.token(32 * w + cols_w - 1), qpos, hi, o);

    // o[mb][q4 * 4 + e] is O^T[channel mb * 32 + q4 * 8 + hi * 4 + e][column n]
    lsum += __shfl_xor(lsum, 32);
    const float inv = 1.0f / lsum;
    if (n < cols_w) {
        __bf16* out = (__bf16*)a.out + row * D + hi * 4;
#pragma unroll
        for (int mb = 0; mb < DT / 32; ++mb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int d = mb * 32 + q4 * 8;
                if (!kExact && d >= D) break;
                tile32::bf16x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[mb][q4 * 4 + e] * inv);
                *reinterpret_cast<tile32::bf16x4*>(out + d) = y;
            }
    }
}

template <int NW, int DT, bool kExact>
ag_status launch(const Args& x, hipStream_t st)
{
    constexpr int lds = lds_bytes(DT);
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> told{0};
        ag_status e = allow_dynamic_lds((const void*)prefill_q8_kernel<NW, DT, kExact>, lds, told);
        if (e) return e;
    }
    const AttnArgs& a = x.a;
    if (a.c.hkv * tiles_bound(a, 32 * NW) + kDealtPast > most_workgroups(64 * NW) || (int64_t)a.total_rows * (a.hq / a.c.hkv) > 0x7fffffff) {
        set_error("too many rows for one launch");
        return AG_ERR_INVALID_ARG;
    }
    const Deal deal = deal_of(a, tiles_bound(a, 32 * NW), std::max(1, stream_cus(st) * (8 / NW) / 8));
    prof_before(st);
    hipLaunchKernelGGL((prefill_q8_kernel<NW, DT, kExact>), dim3((unsigned)workgroups_of(deal)), dim3(64 * NW), lds, st, x, deal);
    prof_after(st);
    return hip_check(hipGetLastError(), "prefill launch");
}

// Few rows on long contexts: the keys of 32 columns dealt to the waves of a workgroup (attn_split_q8.hip) instead of whole tiles, each a chain
// of all of them.  A launch is as long as a chain, or as many as a CU's workgroups come to, and a chain is a start and its share of the
// context; in units of what a context token costs eight waves: 1500 + L, of four 1500 + 2.1 L with two workgroups a CU (three to 96 channels), of tiles 1500 + 4.5 L;
// past 128 channels, one workgroup of one wave a SIMD a CU, of four 1500 + 2.1 L and of tiles 1500 + 9 L; a third more for tiles of 128 or 256 channels where
// attn_split_q8.hip has 96 or 192.  Of several sessions, where more than one round
// evens them out, the mean context is taken for three quarters of the longest.  Graph replay, 32 / 8 heads x 128 unless said otherwise, tiles -> split, us
// (workgroups of 32 columns): one chunk on 6007 tokens of 50 rows (56) 128 -> 32, 211 (216) 133 -> 34, 400 (400) 136 -> 66, 1000 (1000) 150 -> 152; on 2000 of 300 (304) 53 ->
// 27, 1000 72 -> 75; 16 of 30 on 600 (512) 20.4 -> 12.6; 8 of 50..300 on 2000..4000 (1328) 106 -> 100, of 100..200 on 500..1000 (1184) 36 -> 34; 16 of 50..100 on 100..300
// (1248) 19.5 -> 22.1; prompts: 4 of 100 (416) 9.8 -> 7.0, 3 of 250 (768) 13.0 -> 13.1, one of 500 (504) 17.8 -> 9.7, 16 of 200..600 (6568) 58 -> 96; x 64: 211 on 6007 100 -> 26, 8 of
// 50..300 on 2000..4000 73 -> 65, 16 prompts of 200..600 41 -> 50; x 256: 8 of 50..300 on 2000..4000 231 -> 230, 4 of them (696) 161 -> 133, 16 prompts of 200..600 144 -> 240;
// x 96: 8 of 50..300 on 2000..4000 115 -> 76, two prompts of 700 (1408) 25.2 -> 18.2, 16 of 200..600 61 -> 65; x 192: 8 of 100..200 on 500..1000 77 -> 62, two prompts of 700 40.5 -> 49.3.
// fp32 always: tiles with their queries and weights in three terms have one wave a SIMD, and 256 channels spill (eight prompts of 2000 rows x 64 497 -> 457, x 128 782 ->
// 781, x 256 2560 -> 1804; 8 of 100..200 on 500..1000 50 -> 37, 76 -> 59, 225 -> 129).
bool split_preferred(const AttnArgs& a, hipStream_t st)
{
    if (a.c.dtype == AG_F32) return true;
    const int d = a.c.d;
    const bool wide = d > 128;
    const double cus = stream_cus(st), slots = wide ? cus : 2 * cus, few_slots = d <= 96 ? 3 * cus : slots, heads = a.c.hkv, ctx = a.max_ctx, mean = a.batch > 1 ? 0.75 * ctx : ctx;
    const double few = heads * (double)tiles_bound(a, 32), whole = heads * (double)tiles_bound(a, 128);
    const double padding = (d > 64 && d <= 96) || (d > 128 && d <= 192) ? 4.0 / 3 : 1, start = 1500 * padding, step = (wide ? 9 : 4.5) * padding;
    const double split = !wide && few <= cus ? 1500 + ctx : few <= few_slots ? 1500 + 2.1 * ctx : few / few_slots * (1500 + 2.1 * mean);
    const double tiles = whole <= slots ? start + step * ctx : whole / slots * (start + step * mean);
    return split < tiles;
}

// 256 columns a workgroup, bf16 x 128 (at 64 channels eight waves would each bring half a piece a lane, at 256 there are no registers): a tile is
// brought in for twice the columns, but a launch ends on longer chains.  Where the context is
// long, and there are workgroups for two a CU, or one and chunks that are alike beside their contexts.  Graph replay, 128 -> 256 columns, us (of the larger a
// CU): eight prompts of 4096 (16) 1203 -> 1134, 32 chunks of 128..1024 on 2048..8192 (9.5) 1931 -> 1874, of 100..200 on 2000..4000 (2.6) 294 -> 281, two
// of 1000 on 2000 (1) 101 -> 93; but one prompt of 2048 (1) 58 -> 64, eight of 512 (2) 43 -> 48, 64 of 600 (19) 353 -> 380, 16 of 1500 (12) 383 -> 389, one chunk of 1000
// on 6007 (0.5) 150 -> 189.
bool wide_workgroups(const AttnArgs& a, hipStream_t st)
{
    const int64_t cus = stream_cus(st), large = a.c.hkv * tiles_bound(a, 256), ctx = a.max_ctx;
    return ctx > 1536 && (large >= 2 * cus || (large >= cus && ctx >= 2 * (int64_t)a.max_new));
}

}  // namespace

ag_status launch_prefill(const Args& x, hipStream_t st)
{
    if (split_preferred(x.a, st)) return launch_prefill_split(x, st);
    const int d = x.a.c.d;
    if (d == 128 && wide_workgroups(x.a, st)) return launch<8, 128, true>(x, st);
    return d == 64 ? launch<4, 64, true>(x, st) : d < 64 ? launch<4, 64, false>(x, st)
         : d == 128 ? launch<4, 128, true>(x, st) : d < 128 ? launch<4, 128, false>(x, st)
         : d == 256 ? launch<4, 256, true>(x, st) : launch<4, 256, false>(x, st);
}

}  // namespace q8
}  // namespace ag
