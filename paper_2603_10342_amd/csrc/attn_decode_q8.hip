// Decode over the 8-bit paged KV cache: one query per session, any group size, head_dim a multiple of 16 up to 256.
//
// Bound by HBM: 2 Hkv (D + 1) bytes a cached token, read once for all query heads of a KV head.  The schedule is that of the other
// caches' decode: the batch's (session, KV head, block of 16 query heads) pairs are laid end to end in steps - here of 64 tokens, the
// same bytes as 32 of bf16 - and dealt to the workgroups in equal shares (find_share); a share's part of a pair is a segment, whose
// steps the four waves take in contiguous quarters; the segments' (m, l, O) meet in a merge kernel in their order.
//
// A batch of few, short contexts takes one workgroup a pair instead, which writes its result itself.
//
// A wave's step is four 16-token groups, whatever pages they lie in:
//   scores  S^T[token][head]: 16x16x32 bf16 products, rows = 4 slots of each of the 4 groups (product j takes slots 4 j .. 4 j + 3),
//           so that lane group c ends up with all 16 slots of group c - which is what a 16-byte load of the value pool holds
//           of a channel.  The key pool stores four slots of a 16-channel chunk in a run: a load reads 256 contiguous bytes of every group.
//   values  O^T[channel][head] += V^T . P^T, the weights of a lane's 16 slots against 16-byte pieces, slots 0..7 and 8..15.
// Keys and values become bf16 on the way into the products, exactly, two numbers an instruction; a key's power of two goes in
// with that instruction, a value's is multiplied into its weight.
// Two workgroups a CU; three (168 registers, of which 29 are spilled, or the same 198 dealt finer) take 64.3 to 81 us where two take 64 (64 sessions of
// 1024..4096 tokens, 32 / 8 heads x 128, 352 MB: 5.9 TB/s in the split kernel, 4.7 us of merge).  Pages of 64 or 256 instead of 16 change 1 %.
// Weights go into the value product as three bf16 terms, 24 bits, or rounded to bf16 (rounds_weights()); fp32 queries are three terms too.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attn_split_common.h"
#include "q8_internal.h"

namespace ag {
namespace q8 {
namespace {

using splitk::find_share;
using splitk::Share;

constexpr int kTok = 64;                // tokens of a step
constexpr int kWaves = 4;               // of a workgroup
constexpr int kCols = 16;               // query heads of a pair, at most
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ int steps_of(int ctx) { return splitk::steps_of<kTok>(ctx); }
__host__ __device__ inline int blocks_of(int G) { return (G + kCols - 1) / kCols; }

// acc += a . (sum of b's terms), smallest terms first
template <int kTerms>
__device__ __forceinline__ f32x4 product(const bf16x8& a, const bf16x8 (&b)[kTerms], f32x4 acc)
{
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[t], acc, 0, 0, 0);
    return acc;
}

// 64-channel blocks of the keys: the last may be half a one, whose other half is read again, times zeros of the query
constexpr int key_blocks(int dt) { return (dt + 63) / 64; }
template <int DT, bool kExact>
__device__ __forceinline__ int chunk_of(int h, int c, int chunks) { return kExact && DT % 64 == 0 ? 4 * h + c : min(4 * h + c, chunks - 1); }

// fp32 queries are three operands for each of a bf16 one and stand in LDS, as the lanes take them: [block][half][term][lane].  In registers they
// leave one wave a SIMD (16 sessions of 1024..4096 tokens, 32 / 8 heads x 128, 32.0 -> 25.4 us).
template <typename A>
constexpr bool queries_in_lds() { return sizeof(A) == 4; }
template <typename A>
constexpr int query_bytes(int dt) { return queries_in_lds<A>() ? key_blocks(dt) * 2 * terms_of<A>() * 1024 : 0; }

// The queries of heads h0 .. h0 + nh - 1 of (session s, KV head g) as B operands: column = head r, k = channels (4 h + c) * 16 + 8 half .. + 7,
// lane = 16 c + r; zero beyond the heads and channels.
template <typename A, int DT, bool kExact>
__device__ __forceinline__ void query(const AttnArgs& a, int s, int g, int h0, int nh, int lane, int h, int half, bf16x8 (&q)[terms_of<A>()])
{
    const int r = lane & 15, c = lane >> 4, D = kExact ? DT : a.c.d, chunks = D >> 4;
    const A* row = (const A*)a.q + ((int64_t)s * a.hq + (int64_t)g * (a.hq / a.c.hkv) + h0 + min(r, nh - 1)) * D;
    to_terms(row + chunk_of<DT, kExact>(h, c, chunks) * 16 + half * 8, q);
    if (r >= nh || 4 * h + c >= chunks) no_terms(q);
}
template <typename A, int DT, bool kExact>
__device__ __forceinline__ void queries_to_lds(const AttnArgs& a, int s, int g, int h0, int nh, unsigned char* s_q)
{
    constexpr int kTerms = terms_of<A>();
    const int lane = threadIdx.x & 63;
    for (int i = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < 2 * key_blocks(DT); i += kWaves) {
        bf16x8 q[kTerms];
        query<A, DT, kExact>(a, s, g, h0, nh, lane, i >> 1, i & 1, q);
#pragma unroll
        for (int t = 0; t < kTerms; ++t) *reinterpret_cast<bf16x8*>(s_q + (i * kTerms + t) * 1024 + lane * 16) = q[t];
    }
}

// Pages of a step's four groups, by scalar loads: the index is uniform and the table read-only for the kernel's lifetime
struct Ids { int id[4]; };
typedef const __attribute__((address_space(4))) int32_t* cptr_t;
__device__ __forceinline__ Ids pages_of(const AttnArgs& a, int s, int step, int most)
{
    const cptr_t bt = (cptr_t)(uintptr_t)(a.bt + (int64_t)s * a.max_pages);
    Ids p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.id[i] = bt[min((kTok / 16 * step + i) >> (a.c.ps_shift - 4), most)];
    return p;
}

// One wave's part of a segment, steps u0, u0 + kStride .. (n of them) of (session s, KV head g, heads h0 .. h0 + nh - 1 of its group): running maximum,
// this lane's share of the sum, and O^T.  o[mb][i]: channel 16 mb + 4 c + i of head r, lane = 16 c + r.
template <typename A, int DT, bool kExact, int kWeightTerms, int kStride>
__device__ __forceinline__ void attend_steps(const Args& x, int s, int g, int h0, int nh, int ctx, int u0, int n, int lane,
                                             const Ids* first, const unsigned char* s_q, float& m, float& lsum, f32x4 (&o)[DT / 16])
{
    constexpr int kTerms = terms_of<A>(), kH = key_blocks(DT), kV = DT / 16;          // 64-channel blocks of the keys, 16-channel blocks of the values
    const AttnArgs& a = x.a;
    const int D = kExact ? DT : a.c.d, ps = a.c.ps, chunks = D >> 4;
    const int r = lane & 15, c = lane >> 4;
    const float unit = a.scale * kLog2e;
    m = -INFINITY;
    lsum = 0.f;
#pragma unroll
    for (int mb = 0; mb < kV; ++mb) o[mb] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (n <= 0) return;

    bf16x8 q[queries_in_lds<A>() ? 1 : kH][2][kTerms];
    if constexpr (!queries_in_lds<A>()) {
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int half = 0; half < 2; ++half) query<A, DT, kExact>(a, s, g, h0, nh, lane, h, half, q[h][half]);
    }

    const int last_grp = (ctx - 1) >> 4, gshift = a.c.ps_shift - 4, gmask = (1 << gshift) - 1;
    const Finder find(a.c, D, g);
    auto ids_of = [&](int st) { return pages_of(a, s, u0 + st * kStride, last_grp >> gshift); };      // fetched a step before they are used
    // where this lane's group of a step stands: group r / 4 of the keys, c of the values
    auto place = [&](int st, const Ids& p, int mine) {
        Where w = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Where x = find.at(p.id[i], min(4 * (u0 + st * kStride) + i, last_grp) & gmask);
            const uint32_t mask = mine == i ? ~0u : 0u;
            w.data |= x.data & mask;
            w.exps |= x.exps & mask;
        }
        return w;
    };

    u32x4 k[4][kH], v[kV], ve;
    uint32_t ke;
    auto load_k = [&](int st, const Ids& p) {
        const Where w = place(st, p, r >> 2);
        const uint8_t* kp = data_at(a.c.k, w.data) + (r & 3) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int h = 0; h < kH; ++h) {
                k[j][h] = stream16(kp + (j * chunks + chunk_of<DT, kExact>(h, c, chunks)) * 64);
            }
        ke = *reinterpret_cast<const uint32_t*>(exps_at(x.exps, w.exps) + (r & 3) * 4);
    };
    auto load_v = [&](int st, const Ids& p) {
        const Where w = place(st, p, c);
        const uint8_t* vp = data_at(a.c.v, w.data);
#pragma unroll
        for (int mb = 0; mb < kV; ++mb) v[mb] = stream16(vp + (kExact ? mb * 16 + r : min(mb * 16 + r, D - 1)) * 16);
        ve = *reinterpret_cast<const u32x4*>(exps_at(x.exps, w.exps) + ps);
    };

    Ids ids = first && 4 * u0 + 3 <= last_grp ? *first : ids_of(0);
    load_k(0, ids);
    load_v(0, ids);
    ids = ids_of(1);
    __builtin_amdgcn_sched_barrier(0);

    // One step; unless it is the wave's last, the next step's keys are requested as soon as the scores have taken this one's, and
    // its values as soon as the value product has: half a step of every wave is always in flight in the registers of one.
    // Only a wave's last step can reach behind the context.
    auto step = [&](int st, auto last_c) {
        constexpr bool kLast = decltype(last_c)::value;
        f32x4 sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                bf16x8(&qh)[kTerms] = q[queries_in_lds<A>() ? 0 : h][half];
                if constexpr (queries_in_lds<A>()) {
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) qh[t] = *reinterpret_cast<const bf16x8*>(s_q + ((h * 2 + half) * kTerms + t) * 1024 + lane * 16);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sc[j] = product(widen8(k[j][h][2 * half], k[j][h][2 * half + 1], power((ke >> (8 * j)) & 0xFFu)), qh, sc[j]);
            }
        if constexpr (!kLast) {
            __builtin_amdgcn_sched_barrier(0);
            load_k(st + 1, ids);
            __builtin_amdgcn_sched_barrier(0);
        }
        // sc[j][i]: slot 4 j + i of group c
        const int keep = ctx - ((u0 + st * kStride) * kTok + c * 16);      // slot e exists iff e < keep
        float xs[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) xs[e] = !kLast || e < keep ? sc[e >> 2][e & 3] * unit : -INFINITY;
        float mx = xs[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, xs[e]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx);
        const float m_ref = m_new == -INFINITY ? 0.f : m_new;    // (scores that are all -inf or NaN)
        const float alpha = __builtin_amdgcn_exp2f(m - m_ref);
        float psum = 0.f;
        bf16x8 w[2][kWeightTerms];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(xs[half * 8 + i] - m_ref);
            psum = add_weights<kWeightTerms>(psum, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = times_power(p[i], ve, half * 8 + i);
            to_terms(p, w[half]);
        }
        lsum = lsum * alpha + psum;
        if (__builtin_amdgcn_ballot_w64(m_new > m) != 0) {       // (uniform: most steps move no head's maximum)
            asm volatile("");
#pragma unroll
            for (int mb = 0; mb < kV; ++mb) o[mb] *= alpha;
        }
        m = m_new;
        if constexpr (kLast) {                                   // slots behind the last token may hold anything, NaN included
#pragma unroll
            for (int mb = 0; mb < kV; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[mb][i] = keep_bytes(v[mb][i], keep - 4 * i);
        }
#pragma unroll
        for (int mb = 0; mb < kV; ++mb) {
            o[mb] = product(widen8(v[mb][0], v[mb][1], 1.f), w[0], o[mb]);
            o[mb] = product(widen8(v[mb][2], v[mb][3], 1.f), w[1], o[mb]);
        }
        if constexpr (!kLast) {
            __builtin_amdgcn_sched_barrier(0);
            load_v(st + 1, ids);
            ids = ids_of(st + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll 1
    for (int st = 0; st + 1 < n; ++st) step(st, std::false_type{});
    step(n - 1, std::true_type{});
}

// LDS of a workgroup: per wave and head O, then m and l
inline size_t lds_of(int nh, int d) { return (size_t)kWaves * nh * (d + 2) * sizeof(float); }

// A wave's results of a pair's nh heads into LDS (s_o: [wave][head][D], then m and l [wave][head], `rows` heads a wave) ...
template <int DT, bool kExact>
__device__ __forceinline__ void results_to_lds(float* s_o, int w, int rows, int nh, int D, int lane, float m, float lsum, const f32x4 (&o)[DT / 16])
{
    const int r = lane & 15, c = lane >> 4;
    float* const s_m = s_o + kWaves * rows * D;
    if (r < nh) {
#pragma unroll
        for (int mb = 0; mb < DT / 16; ++mb)
            if (kExact || mb * 16 < D) *reinterpret_cast<f32x4*>(s_o + (w * rows + r) * D + mb * 16 + c * 4) = o[mb];
        if (c == 0) { s_m[w * rows + r] = m; s_m[(kWaves + w) * rows + r] = lsum; }
    }
}
// ... and the waves' together, of four channels of a head.
__device__ __forceinline__ f32x4 combine(const float* s_o, int rows, int D, int head, int d, float& ms, float& l)
{
    const float* const s_m = s_o + kWaves * rows * D;
    ms = s_m[head];
#pragma unroll
    for (int ww = 1; ww < kWaves; ++ww) ms = fmaxf(ms, s_m[ww * rows + head]);
    const float ref = ms == -INFINITY ? 0.f : ms;
    l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < kWaves; ++ww) {
        const float fw = __builtin_amdgcn_exp2f(s_m[ww * rows + head] - ref);         // a wave without steps has m = -inf -> 0
        const f32x4 y = *reinterpret_cast<const f32x4*>(s_o + (ww * rows + head) * D + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += fw * y[e];
        l += fw * s_m[(kWaves + ww) * rows + head];
    }
    return acc;
}

template <typename A, int DT, bool kExact, int kWeightTerms>
__global__ __launch_bounds__(64 * kWaves, DT > 128 ? 1 : 2) void decode_q8_split_kernel(Args x, int32_t* __restrict__ hdr, float* __restrict__ ws_o,
                                                                                                          float* __restrict__ ws_ml, int pmax)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char s_q[];   // queries, then the waves' results
    float* const s_o = reinterpret_cast<float*>(s_q + query_bytes<A>(DT));            // [wave][head][D], then m and l [wave][head]
    const AttnArgs& a = x.a;
    const int B = a.batch, hkv = a.c.hkv, hq = a.hq, G = hq / hkv, D = kExact ? DT : a.c.d;
    const int nb = blocks_of(G), pairs = hkv * nb, rows = min(G, kCols);
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wg = blockIdx.x;

    Share sh;
    if (!find_share<true, kTok>(a.ctx_lens, B, pairs, hdr, sh)) return;
    const int q = sh.q, f1 = sh.f1;
    int s = sh.s, base = sh.base, ctx = sh.ctx, n = steps_of(ctx);
    int pair = (sh.f0 - base) / n;
    int u = (sh.f0 - base) - pair * n;
    for (int f = sh.f0; f < f1 && s < B;) {               // one segment per pass; every value here is uniform
        const int k = min(n - u, f1 - f);                 // steps of this segment
        if (k <= 0) break;                                // (only if the lengths changed under the kernel: never spin)
        const int per = (k + kWaves - 1) / kWaves;
        const int g = pair / nb, h0 = (pair - g * nb) * kCols, nh = min(G - h0, kCols);
        float m, lsum;
        f32x4 o[DT / 16];
        if constexpr (queries_in_lds<A>()) {
            queries_to_lds<A, DT, kExact>(a, s, g, h0, nh, s_q);
            __syncthreads();
        }
        attend_steps<A, DT, kExact, kWeightTerms, 1>(x, s, g, h0, nh, ctx, u + w * per, max(0, min(per, k - w * per)), lane, nullptr, s_q, m, lsum, o);
        lsum += __shfl_xor(lsum, 16);
        lsum += __shfl_xor(lsum, 32);
        results_to_lds<DT, kExact>(s_o, w, rows, nh, D, lane, m, lsum, o);
        __syncthreads();
        // the pair starts at flat step base + pair n; its segments are numbered from the workgroup holding that step
        const int piece = wg - (base + pair * n) / q;
        if (piece < pmax) {
            for (int idx = tid; idx < nh * (D / 4); idx += 64 * kWaves) {      // four channels a thread
                const int head = idx / (D / 4), d = (idx - head * (D / 4)) * 4;
                float ms, l;
                const f32x4 acc = combine(s_o, rows, D, head, d, ms, l);
                const int64_t slot = ((int64_t)s * hq + (int64_t)g * G + h0 + head) * pmax + piece;
                *reinterpret_cast<f32x4*>(ws_o + slot * D + d) = acc;
                if (d == 0) { ws_ml[slot * 2] = ms; ws_ml[slot * 2 + 1] = l; }
            }
        }
        __syncthreads();                                  // s_o is rewritten by the next segment
        f += k;
        u += k;
        if (u == n) {                                     // on to the next pair
            u = 0;
            if (++pair == pairs) {
                pair = 0;
                base += pairs * n;
                do {
                    ++s;
                    ctx = s < B ? a.ctx_lens[s] : 0;
                    n = steps_of(ctx);
                } while (s < B && n == 0);
            }
        }
    }
}

// A batch of few, short contexts: one workgroup a pair, which writes its result itself - no plan, no partials, no merge, whose dependent
// round trips are most of a small step.  Four waves and two workgroups a CU: eight are no faster alone (one session of 500 to 1000 tokens 7.8 us, four
// 7.5) and leave room for half as many pairs (256 sessions of 1 to 512 46 us, four 29).  Beside the split kernel's loop, whose steps follow one another, this
// one holds about 50 registers more (239 of them for 188 at 128 channels, one term): two waves a SIMD instead of three at 96, and spills at padded widths - 12 registers at 112
// channels, 45 at 208 to 240, with fp32 queries 4 and 3 (240 channels, 64 sessions of 1 to 512 27.8 us, with one term and 29 spilled 24.0).

template <typename A, int DT, bool kExact, int kWeightTerms>
__global__ __launch_bounds__(64 * kWaves, DT > 128 ? 1 : 2) void decode_q8_direct_kernel(Args x)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char s_q[];   // as in the split kernel
    float* const s_o = reinterpret_cast<float*>(s_q + query_bytes<A>(DT));
    const AttnArgs& a = x.a;
    const int hkv = a.c.hkv, hq = a.hq, G = hq / hkv, D = kExact ? DT : a.c.d;
    const int nb = blocks_of(G), pairs = hkv * nb, rows = min(G, kCols);
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = blockIdx.x / pairs, pair = blockIdx.x - s * pairs, g = pair / nb, h0 = (pair - g * nb) * kCols, nh = min(G - h0, kCols);
    // the first step's pages beside the length, as a wave's steps are every fourth one whatever that is: a round trip
    // less (one session of 1000 tokens 8.8 -> 8.3 us, of 500 6.3 -> 6.1)
    const Ids first = pages_of(a, s, w, a.max_pages - 1);
    const int ctx = a.ctx_lens[s];
    asm volatile("" :: "s"(ctx), "s"(first.id[0]), "s"(first.id[1]), "s"(first.id[2]), "s"(first.id[3]));
    A* const out = (A*)a.out + ((int64_t)s * hq + (int64_t)g * G + h0) * D;
    if (ctx <= 0) {                     // uniform over the workgroup
        for (int idx = tid; idx < nh * D; idx += 64 * kWaves) out[idx] = (A)0.0f;
        return;
    }
    const int n = steps_of(ctx);
    float m, lsum;
    f32x4 o[DT / 16];
    if constexpr (queries_in_lds<A>()) {
        queries_to_lds<A, DT, kExact>(a, s, g, h0, nh, s_q);
        __syncthreads();
    }
    attend_steps<A, DT, kExact, kWeightTerms, kWaves>(x, s, g, h0, nh, ctx, w, max(0, (n - w + kWaves - 1) / kWaves), lane, &first, s_q, m, lsum, o);
    lsum += __shfl_xor(lsum, 16);
    lsum += __shfl_xor(lsum, 32);
    results_to_lds<DT, kExact>(s_o, w, rows, nh, D, lane, m, lsum, o);
    __syncthreads();
    for (int idx = tid; idx < nh * (D / 4); idx += 64 * kWaves) {
        const int head = idx / (D / 4), d = (idx - head * (D / 4)) * 4;
        float ms, l;
        const f32x4 acc = combine(s_o, rows, D, head, d, ms, l);
        const float y[4] = {acc[0] / l, acc[1] / l, acc[2] / l, acc[3] / l};
        splitk::store_quad(out + head * D + d, y);
    }
}

// D / 4 lanes per (session, query head), `rows` of them a workgroup.  The first four partials, the plan and the context's length are fetched
// together, before anything says how many there are: one memory round trip instead of three, of which this launch consists.  Further ones come
// eight at a time (one session of 16000 tokens, 32 partials: 18.2 -> 16.2 us).
template <typename A>
__global__ __launch_bounds__(256) void decode_q8_merge_kernel(Args x, const int32_t* __restrict__ hdr, const float* __restrict__ ws_o,
                                                              const float* __restrict__ ws_ml, int pmax, int rows)
{
    const AttnArgs& a = x.a;
    const int D = a.c.d, G = a.hq / a.c.hkv, nb = blocks_of(G);
    const int mine = threadIdx.x / (D / 4);
    const int64_t row = (int64_t)blockIdx.x * rows + mine;             // s * hq + h
    if (mine >= rows || row >= (int64_t)a.batch * a.hq) return;
    const int s = (int)(row / a.hq), h = (int)(row - (int64_t)s * a.hq), d = (threadIdx.x - mine * (D / 4)) * 4;
    const float* const po = ws_o + row * pmax * D + d;
    const float* const pml = ws_ml + row * pmax * 2;
    const int ctx = a.ctx_lens[s], share = hdr[0], before = hdr[1 + s];
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    int pieces = 0;
    // partials first .. first + N - 1, in their order (those that were not written hold anything: not used)
    auto take = [&](int first, auto count, auto known) {
        constexpr int N = decltype(count)::value;
        float ml[N][2];
        f32x4 y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t at = min(first + i, pmax - 1);
            ml[i][0] = pml[at * 2];
            ml[i][1] = pml[at * 2 + 1];
            y[i] = *reinterpret_cast<const f32x4*>(po + at * D);
        }
        known();
        float m_new = m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (first + i >= pieces) ml[i][0] = -INFINITY;
            m_new = fmaxf(m_new, ml[i][0]);
        }
        const float ref = m_new == -INFINITY ? 0.f : m_new, keep = __builtin_amdgcn_exp2f(m - ref);
        l *= keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= keep;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (first + i < pieces) {
                const float f = __builtin_amdgcn_exp2f(ml[i][0] - ref);
                l += f * ml[i][1];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += f * y[i][e];
            }
        }
        m = m_new;
    };
    take(0, std::integral_constant<int, 4>{}, [&] {
        if (ctx <= 0) return;
        const int g = h / G, pair = g * nb + (h - g * G) / kCols;
        const int q = max(1, share), n = steps_of(ctx);
        const int first = a.c.hkv * nb * before + pair * n;            // the pair's first flat step
        pieces = min(pmax, (first + n - 1) / q - first / q + 1);
    });
    for (int first = 4; first < pieces; first += 8) take(first, std::integral_constant<int, 8>{}, [] {});
    const float inv = pieces > 0 ? 1.f / l : 0.f;                      // (a session without context: zeros)
    const float r[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    splitk::store_quad((A*)a.out + row * D + d, r);
}

struct Partials { int32_t* hdr; float *o, *ml; int pmax; };

// grid: workgroups of the split kernel, or 0 for one workgroup a pair
template <typename A, int DT, bool kExact, int kWeightTerms = 3>
ag_status launch(const Args& x, const Partials& p, int grid, hipStream_t st)
{
    const AttnArgs& a = x.a;
    const int G = a.hq / a.c.hkv;
    const size_t lds = query_bytes<A>(DT) + lds_of(std::min(G, kCols), a.c.d);
    if (lds > 64 * 1024) {
        static std::atomic<uint64_t> told[2] = {};
        const void* kernel = grid ? (const void*)decode_q8_split_kernel<A, DT, kExact, kWeightTerms> : (const void*)decode_q8_direct_kernel<A, DT, kExact, kWeightTerms>;
        ag_status e = allow_dynamic_lds(kernel, query_bytes<A>(DT) + (int)lds_of(kCols, DT), told[grid ? 0 : 1]);
        if (e) return e;
    }
    if (grid) hipLaunchKernelGGL((decode_q8_split_kernel<A, DT, kExact, kWeightTerms>), dim3(grid), dim3(64 * kWaves), lds, st, x, p.hdr, p.o, p.ml, p.pmax);
    else hipLaunchKernelGGL((decode_q8_direct_kernel<A, DT, kExact, kWeightTerms>), dim3(a.batch * a.c.hkv * blocks_of(G)), dim3(64 * kWaves), lds, st, x);
    return hip_check(hipGetLastError(), "decode launch");
}

// Decode keeps of a softmax weight what it keeps over a bf16 cache of the same shape (ag.h): all 24 bits, but for bf16 with 128 channels on pages
// of 16 and up to 16 heads a group, where it is rounded to bf16, off by up to 2^-8 of itself, independently of the others.  Three terms there: one session
// of 1000 tokens 8.2 -> 9.6 us, 64 of 1 to 512 9.4 -> 10.3, 64 of 1024 to 4096 63.3 -> 64.3.  One term elsewhere: 64 sessions of 1000 to 2000 x 64 19.2 -> 18.2 us, x 256
// 75.5 -> 73.7.
bool rounds_weights(const AttnArgs& a) { return a.c.dtype == AG_BF16 && a.c.d == 128 && a.c.ps == 16 && a.hq <= kCols * a.c.hkv; }

// The least of five widths that holds a head: 96 channels in 128 are 25 to 30 % slower (64 sessions of 1000..2000 tokens 36.5 us, 27.7; of 1..512 11.4, 9.1), 192 in 256 20 % (70.3,
// 58.1).
template <typename A>
ag_status launch_typed(const Args& x, const Partials& p, int grid, hipStream_t st)
{
    const int d = x.a.c.d;
    if constexpr (sizeof(A) == 2) {
        if (rounds_weights(x.a)) return launch<A, 128, true, 1>(x, p, grid, st);
    }
    return d == 64 ? launch<A, 64, true>(x, p, grid, st) : d < 64 ? launch<A, 64, false>(x, p, grid, st)
         : d == 96 ? launch<A, 96, true>(x, p, grid, st) : d < 96 ? launch<A, 96, false>(x, p, grid, st)
         : d == 128 ? launch<A, 128, true>(x, p, grid, st) : d < 128 ? launch<A, 128, false>(x, p, grid, st)
         : d == 192 ? launch<A, 192, true>(x, p, grid, st) : d < 192 ? launch<A, 192, false>(x, p, grid, st)
         : d == 256 ? launch<A, 256, true>(x, p, grid, st) : launch<A, 256, false>(x, p, grid, st);
}

int merge_rows(const AttnArgs& a) { return 256 / (a.c.d / 4); }
int64_t merge_workgroups(const AttnArgs& a) { return ((int64_t)a.batch * a.hq + merge_rows(a) - 1) / merge_rows(a); }

template <typename A>
ag_status launch_merge(const Args& x, const Partials& p, hipStream_t st)
{
    const int rows = merge_rows(x.a);
    hipLaunchKernelGGL(decode_q8_merge_kernel<A>, dim3((unsigned)merge_workgroups(x.a)), dim3(256), 0, st, x, p.hdr, p.o, p.ml, p.pmax, rows);
    return hip_check(hipGetLastError(), "decode merge launch");
}

// A workgroup alone takes 2 us for every 256 tokens, with fp32 queries 2.6, and the longest pair's is the least a launch takes (the host
// knows no other length); shares take about 10 whatever the context of few pairs, and a segment each - 2.5 us - for short pairs one after
// the other.  Past half of the CUs a pair each keeps them busy anyway; long contexts are left to shares, as one among short ones would be
// all that a launch waits for.  Graph replay, shares -> one workgroup a pair, us (pairs at 256 CUs), 8 KV heads, x 128 on pages of 16: one session of 1000 tokens (8) 9.4 ->
// 8.5, 1600 (8) 11.9 -> 12.5, 2400 (8) 12.7 -> 16.2, 8 of 1000 (64) 9.9 -> 9.6, 16 of 1600 (128) 16.8 -> 14.5, 32 of 2400 (256) 29.3 -> 26.4, of 500 to 4000 (256) 30.2 -> 29.0, 64 of 1 to
// 128 (512) 25.4 -> 6.2, of 1 to 512 27.5 -> 10.0, of 1000 to 2000 39.0 -> 33.5, of 1024 to 4096 63.9 -> 62.5, 256 of 1000 to 2000 (2048) 142 -> 127; weights in 24 bits, pages of 32: one of
// 1000 9.9 -> 10.3, 1600 12.8 -> 14.5, 64 of 1000 to 2000 38.5 -> 35.5; x 64: one of 1600 10.6 -> 10.5, 2400 12.0 -> 14.7, 64 of 1000 to 2000 24.0 -> 20.4; x 96: one of 1000 9.4 -> 9.0, 64 of
// 1000 to 2000 31.5 -> 28.1; x 256: one of 500 13.4 -> 10.9, 1000 13.3 -> 16.3, 64 of 1000 to 2000 75.9 -> 71.5; fp32 x 128: one of 1000 10.9 -> 11.7, 16 of 1600 20.0 -> 18.0, 64 of 1000 to 2000
// 40.8 -> 37.4, 16 of 1024 to 4096 24.8 -> 32.7.
bool one_workgroup_a_pair(const AttnArgs& a, int64_t pairs, int64_t cus)
{
    const int64_t size = (int64_t)a.max_ctx * (a.c.d + 64), line = a.c.dtype == AG_BF16 ? 400000 : 290000;
    return pairs <= most_workgroups(64 * kWaves) && 8 * size <= (2 * pairs > cus ? 8 : 5) * line;
}

}  // namespace

size_t decode_workspace(int batch, int hq, int d, int max_ctx)
{
    return splitk::header_ints(batch) * sizeof(int32_t) + (size_t)batch * hq * splitk::pieces_max<kTok>(max_ctx) * (size_t)(d + 2) * sizeof(float);
}

ag_status launch_decode(const Args& x, void* ws, hipStream_t st)
{
    const AttnArgs& a = x.a;
    const bool bf16 = a.c.dtype == AG_BF16;
    const int64_t pairs = (int64_t)a.c.hkv * blocks_of(a.hq / a.c.hkv) * a.batch;
    Partials p;
    p.pmax = splitk::pieces_max<kTok>(a.max_ctx);
    p.hdr = (int32_t*)ws;
    p.o = (float*)(p.hdr + splitk::header_ints(a.batch));
    p.ml = p.o + (size_t)a.batch * a.hq * p.pmax * a.c.d;
    ag_status e = AG_OK;
    if (a.max_ctx > 0 && one_workgroup_a_pair(a, pairs, stream_cus(st))) {
        prof_before(st);
        e = bf16 ? launch_typed<__bf16>(x, p, 0, st) : launch_typed<float>(x, p, 0, st);
        prof_after(st);
        return e;
    }
    // Upper bound of the step count from the host-known bounds: a share is at most kMaxSteps steps even if every session is max_ctx long.
    const int64_t f_max = pairs * ((a.max_ctx + (kTok - 1)) / kTok);
    if (f_max > (1 << 30)) { set_error("decode batch of %lld steps of %d tokens is beyond one launch", (long long)f_max, kTok); return AG_ERR_INVALID_ARG; }
    if (merge_workgroups(a) > most_workgroups(256)) { set_error("decode batch of %lld rows is beyond one launch", (long long)a.batch * a.hq); return AG_ERR_INVALID_ARG; }
    prof_before(st);
    if (a.max_ctx > 0) e = bf16 ? launch_typed<__bf16>(x, p, share_workgroups(f_max, st), st) : launch_typed<float>(x, p, share_workgroups(f_max, st), st);
    if (!e) e = bf16 ? launch_merge<__bf16>(x, p, st) : launch_merge<float>(x, p, st);
    prof_after(st);
    return e;
}

}  // namespace q8
}  // namespace ag
