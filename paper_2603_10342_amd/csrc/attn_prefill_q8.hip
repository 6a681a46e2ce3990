// Cold and resume prefill over the 8-bit paged KV cache: causal attention of ragged chunks behind cached prefixes, any group
// size, head_dim a multiple of 16 up to 256.
//
// A dense contraction, bound by the matrix cores.  A workgroup of NW waves owns 32 * NW columns of one (session, KV head), a
// column being a (token, query head of the group) pair; a wave owns 32 of them with their queries in registers, and takes keys and
// values 64 at a time in the tile arithmetic of the bf16 caches (attn_tile32.h).  What differs is how a tile comes into LDS:
// its bytes go through registers, one tile ahead, and are written as bf16 numbers, their powers of two multiplied in (exactly).
// Done once a workgroup that is an eighth (NW = 8) of what a conversion behind LDS would cost each wave, and the products run as
// they do over a bf16 cache.  A wave brings one 16-token group of the tile (or half of one): one page id, 16 exponent bytes.
//   iteration t: K(t + 1) and V(t) from registers into LDS; K(t + 2) and V(t + 1) requested; S(t) = K(t) Q^T; P(t) side by side with
//   O += V(t - 1) P(t - 1); barrier.
// bf16 activations: weights rounded to bf16 for the value product; fp32: queries and weights as three bf16 terms.
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

template <typename A>
constexpr int terms_of() { return sizeof(A) == 4 ? 3 : 1; }
// two key and two value tiles
constexpr int lds_bytes(int dt) { return 4 * tile_bytes(dt); }

__device__ __forceinline__ void query_terms(const __bf16* p, bf16x8 (&t)[1]) { t[0] = *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ void query_terms(const float* p, bf16x8 (&t)[3])
{
    const Terms x = split8(*reinterpret_cast<const Four*>(p), *reinterpret_cast<const Four*>(p + 4));
    t[0] = __builtin_bit_cast(bf16x8, x.h);
    t[1] = __builtin_bit_cast(bf16x8, x.m);
    t[2] = __builtin_bit_cast(bf16x8, x.l);
}

// S^T tile = K tile . Q^T with queries in terms, smallest first (one term: tile32::qk_tile)
template <int DT, int kTerms>
__device__ __forceinline__ void scores(const unsigned char* kb, const bf16x8 (&q)[DT / 16][kTerms], f32x16 (&sc)[2])
{
    constexpr int kAhead = tile32::kOperandsAhead, kN = DT / 8;
    bf16x8 opnd[kAhead + 1];
    auto operand = [&](int i) -> const unsigned char* { return kb + (i & 1) * 512 + (i >> 1) * 2048; };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) opnd[i] = *reinterpret_cast<const bf16x8*>(operand(i));
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        if (i + kAhead < kN) opnd[(i + kAhead) % (kAhead + 1)] = *reinterpret_cast<const bf16x8*>(operand(i + kAhead));
#pragma unroll
        for (int t = kTerms - 1; t >= 0; --t)
            sc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(opnd[i % (kAhead + 1)], q[i >> 1][t], i < 2 && t == kTerms - 1 ? zero : sc[i & 1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// An iteration's vector work and value product one after the other: at 256 channels, where there are two products to a score and
// nothing is gained by laying them side by side (tile32::softmax_and_value_product).
template <int DT, bool kLo>
__device__ __forceinline__ void softmax_after_value_product(bool do_sm, bool do_pv, const unsigned char* vb, const f32x16 (&sc)[2], float sl2, float& m,
                                                            float& lsum, const Weights<kLo>& p_prev, Weights<kLo>& p_cur, f32x16 (&o)[DT / 32])
{
    if (do_pv) tile32::pv_tile<DT, kLo>(vb, p_prev, o);
    if (!do_sm) return;
    float mx = tile32::row_max(sc) * sl2;
    // m is shared by the two lanes of a query: if either lane's own maximum outgrew it, combine them
    if (__builtin_amdgcn_ballot_w64(mx > m + tile32::kRescaleSlack) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        lsum *= alpha;
#pragma unroll
        for (int mb = 0; mb < DT / 32; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mb][i] *= alpha;
        m = m_new;
    }
    tile32::exp_tile<kLo>(sc, sl2, m == -INFINITY ? 0.f : m, lsum, p_cur);
}

template <typename A, int NW, int DT, bool kExact>
__global__ __launch_bounds__(64 * NW, DT > 128 || sizeof(A) == 4 ? 1 : 2) void prefill_q8_kernel(Args x, Deal deal)
{
    constexpr int kTerms = terms_of<A>();
    constexpr bool kLo = kTerms > 1;
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
    const int col = min(32 * w + n, cols - 1);                                // columns beyond the tile repeat the last one
    const int token = columns.token(col), head = columns.head(col, token);
    const int qpos = P + token;
    const int64_t row = ((int64_t)row0 + token) * hq + (int64_t)g * G + head;

    // ---- tile requests: this wave's group of the tile, 16 keys; pieces [chunk][key] of the keys, [channel] of the values ----
    typedef const __attribute__((address_space(4))) int32_t* cptr_t;
    const cptr_t bt = (cptr_t)(uintptr_t)(a.bt + (int64_t)s * a.max_pages);
    const int last_grp = (ctx - 1) >> 4, gshift = a.c.ps_shift - 4, gmask = (1 << gshift) - 1;
    const int64_t block = (int64_t)D * ps;                                    // bytes of one (page, head)
    const int my_grp = w / kWavesPerGroup, piece0 = (w % kWavesPerGroup) * kPer * 64 + lane;
    const int key = lane & 15;                                                // of the group, in every piece of a lane
    const uint8_t* const kpool = (const uint8_t*)a.c.k;
    const uint8_t* const vpool = (const uint8_t*)a.c.v;
    u32x4 kr[kPer], vr[kPer], ve = {0, 0, 0, 0};
    uint32_t ke = 0;
    auto page_of = [&](int t) { return bt[min(t * 4 + my_grp, last_grp) >> gshift]; };
    auto request_k = [&](int t, int page) {
        const int gi = min(t * 4 + my_grp, last_grp) & gmask;
        const int64_t at = (int64_t)page * hkv + g;
        const uint8_t* kp = kpool + at * block + gi * 16 * D + (key >> 2) * chunks * 64 + (key & 3) * 16;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int chunk = (piece0 + i * 64) >> 4;
            kr[i] = u32x4{0, 0, 0, 0};
            if (kExact || chunk < chunks) kr[i] = *reinterpret_cast<const u32x4*>(kp + chunk * 64);
        }
        ke = x.exps[at * (2 * ps) + gi * 16 + key_place(key)];
    };
    auto request_v = [&](int t, int page) {
        const int gi = min(t * 4 + my_grp, last_grp) & gmask;
        const int64_t at = (int64_t)page * hkv + g;
        const uint8_t* vp = vpool + at * block + gi * 16 * D;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int ch = piece0 + i * 64;
            vr[i] = u32x4{0, 0, 0, 0};
            if (kExact || ch < D) vr[i] = *reinterpret_cast<const u32x4*>(vp + ch * 16);
        }
        ve = *reinterpret_cast<const u32x4*>(x.exps + at * (2 * ps) + ps + gi * 16);
    };
    // into LDS as bf16: K [chunk of 8 channels][64 keys], V [chunk of 8 keys][channel], 16-byte pieces
    auto put_k = [&](int t) {
        unsigned char* dst = lds + (t & 1) * kTile + (my_grp * 16 + key) * 16;
        const float scale = power(ke);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int chunk = (piece0 + i * 64) >> 4;
            *reinterpret_cast<bf16x8*>(dst + chunk * 2048) = widen8(kr[i][0], kr[i][1], scale);
            *reinterpret_cast<bf16x8*>(dst + chunk * 2048 + 1024) = widen8(kr[i][2], kr[i][3], scale);
        }
    };
    auto put_v = [&](int t) {
        unsigned char* dst = lds + (2 + (t & 1)) * kTile + my_grp * (DT * 32);
        const int keep = ctx - (t * BN + my_grp * 16);       // slots behind the last token may hold anything, NaN included: zeros
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = power_of(ve, i);
        if (keep < 16) {                                     // uniform
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] = i < keep ? e[i] : 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) vr[i][k] = keep_bytes(vr[i][k], keep - 4 * k);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int ch = piece0 + i * 64;
#pragma unroll
            for (int half = 0; half < 2; ++half) {           // slots half * 4 + {0..3} and 8 + half * 4 + {0..3}
                u32x4 y;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int o = half * 4 + k * 8;
                    y[2 * k] = widen_pair<false>(vr[i][half + 2 * k], e[o], e[o + 1]);
                    y[2 * k + 1] = widen_pair<true>(vr[i][half + 2 * k], e[o + 2], e[o + 3]);
                }
                *reinterpret_cast<u32x4*>(dst + half * (DT * 16) + ch * 16) = y;
            }
        }
    };

    request_k(0, page_of(0));

    // ---- Q^T as B operand: column n, k-step ks covers channels ks * 16 + hi * 8 .. + 7 ----
    bf16x8 qf[DT / 16][kTerms];
    {
        const A* qp = (const A*)a.q + row * D + hi * 8;
#pragma unroll
        for (int ks = 0; ks < DT / 16; ++ks) {
            if (kExact || ks < chunks) {
                query_terms(qp + ks * 16, qf[ks]);
            } else {
#pragma unroll
                for (int t = 0; t < kTerms; ++t) qf[ks][t] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
        }
    }
    const float sl2 = a.scale * tile32::kLog2e;
    float m = -INFINITY, lsum = 0.f;
    f32x16 o[DT / 32];
#pragma unroll
    for (int mb = 0; mb < DT / 32; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[mb][i] = 0.f;

    put_k(0);
    request_v(0, page_of(0));
    request_k(min(1, n_tiles - 1), page_of(min(1, n_tiles - 1)));
    __syncthreads();

    const unsigned char* const k_lane = lds + n * 16 + hi * 1024;
    const unsigned char* const v_lane = lds + 2 * kTile + n * 16 + hi * (DT * 16);
    f32x16 sc[2];
    Weights<kLo> pa, pb;
    // Requests past the last tile repeat it; what they bring is written to a place that nobody reads.
    auto iter = [&](int t, Weights<kLo>& p_prev, Weights<kLo>& p_cur) {
        put_k(t + 1);
        put_v(t);
        const int tk = min(t + 2, n_tiles - 1), tv = min(t + 1, n_tiles - 1);
        request_k(tk, page_of(tk));
        request_v(tv, page_of(tv));
        const bool do_sm = t < wave_tiles, do_pv = t >= 1 && t - 1 < wave_tiles;
        const unsigned char* kb = k_lane + (t & 1) * kTile;
        const unsigned char* vb = v_lane + ((t + 1) & 1) * kTile;             // V(t - 1)
        if (do_sm) {
            scores<DT, kTerms>(kb, qf, sc);
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
        }
        if constexpr (DT > 128) softmax_after_value_product<DT, kLo>(do_sm, do_pv, vb, sc, sl2, m, lsum, p_prev, p_cur, o);
        else tile32::softmax_and_value_product<DT, kLo>(do_sm, do_pv, vb, sc, sl2, m, lsum, p_prev, p_cur, o);
        __syncthreads();
    };
#pragma unroll 1
    for (int t = 0; t <= n_tiles; t += 2) {
        iter(t, pb, pa);
        if (t + 1 <= n_tiles) iter(t + 1, pa, pb);
    }

    // o[mb][q4 * 4 + e] is O^T[channel mb * 32 + q4 * 8 + hi * 4 + e][column n]
    lsum += __shfl_xor(lsum, 32);
    const float inv = 1.0f / lsum;
    if (n < cols_w) {
        A* out = (A*)a.out + row * D + hi * 4;
        typedef A quad __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int mb = 0; mb < DT / 32; ++mb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int d = mb * 32 + q4 * 8;
                if (!kExact && d >= D) break;
                quad y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (A)(o[mb][q4 * 4 + e] * inv);
                *reinterpret_cast<quad*>(out + d) = y;
            }
    }
}

// sum_s ceil(N_s G / cols) <= total G / cols + batch, and no session has more than ceil(max_new G / cols)
int64_t tiles_bound(const AttnArgs& a, int cols)
{
    const int64_t G = a.hq / a.c.hkv;
    return std::min<int64_t>((int64_t)a.total_rows * G / cols + a.batch, (int64_t)a.batch * ((a.max_new * G + cols - 1) / cols));
}

template <typename A, int NW, int DT, bool kExact>
ag_status launch(const Args& x, hipStream_t st)
{
    constexpr int lds = lds_bytes(DT);
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> told{0};
        ag_status e = allow_dynamic_lds((const void*)prefill_q8_kernel<A, NW, DT, kExact>, lds, told);
        if (e) return e;
    }
    const AttnArgs& a = x.a;
    if (a.c.hkv * tiles_bound(a, 32 * NW) + kDealtPast > 0x7fffffff || (int64_t)a.total_rows * (a.hq / a.c.hkv) > 0x7fffffff) {
        set_error("too many rows for one launch");
        return AG_ERR_INVALID_ARG;
    }
    const Deal deal = deal_of(a, tiles_bound(a, 32 * NW), std::max(1, stream_cus(st) * (8 / NW) / 8));
    prof_before(st);
    hipLaunchKernelGGL((prefill_q8_kernel<A, NW, DT, kExact>), dim3((unsigned)workgroups_of(deal)), dim3(64 * NW), lds, st, x, deal);
    prof_after(st);
    return hip_check(hipGetLastError(), "prefill launch");
}

template <typename A>
ag_status launch_typed(const Args& x, hipStream_t st)
{
    const int d = x.a.c.d;
    return d == 64 ? launch<A, 4, 64, true>(x, st) : d < 64 ? launch<A, 4, 64, false>(x, st)
         : d == 128 ? launch<A, 4, 128, true>(x, st) : d < 128 ? launch<A, 4, 128, false>(x, st)
         : d == 256 ? launch<A, 4, 256, true>(x, st) : launch<A, 4, 256, false>(x, st);
}

}  // namespace

ag_status launch_prefill(const Args& x, hipStream_t st)
{
    return x.a.c.dtype == AG_BF16 ? launch_typed<__bf16>(x, st) : launch_typed<float>(x, st);
}

}  // namespace q8
}  // namespace ag
