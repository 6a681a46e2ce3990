// Prefill of few rows over the 8-bit paged KV cache, and of any number with fp32 activations: the keys of 32 columns - (token, query head of the group) pairs of one (session, KV
// head) - are dealt to the waves of one workgroup, whose sums meet in LDS.
//
// A chunk of a few hundred rows on a long context makes few workgroups of whole tiles, each a chain of as many key tiles as the context has
// (attn_prefill_q8.hip).  Here a chain is a W-th of that.  No wave shares a tile with another, so nothing goes through LDS: keys
// and values come from the pools straight into the operands of 32x32x16 bf16 products, converted in registers.  A step of a wave is 32
// keys, two 16-token groups:
//   scores  S^T[key][column]: row n is slot 4 (n / 8) + n % 4 of group (n / 4) % 2, so that a lane ends up with the 16 slots of group
//           hi = lane / 32, which are the 16 bytes that a load of the value pool holds of a channel; a key's power goes in with the conversion
//   values  O^T[channel][column] += V^T . P^T: slots 0..7 and 8..15 of the lane's group; a value's power is multiplied into its weight.  With bf16
//           activations that is rounded to bf16, as in whole tiles (attn_prefill_q8.hip; in three terms 211 rows on 6007 tokens 35 -> 50 us, x 64 24 -> 36)
// The next step's keys are requested when the scores have taken this one's, its values when the value product has.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "q8_internal.h"
#include "tile_list.h"

namespace ag {
namespace q8 {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTok = 32;                // keys of a step
constexpr int kCols = 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;          // a reference maximum may be outgrown by 2^8 before O is rescaled

template <int kTerms>
__device__ __forceinline__ f32x16 product(const bf16x8& a, const bf16x8 (&b)[kTerms], f32x16 acc)
{
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b[t], acc, 0, 0, 0);
    return acc;
}

// fp32 queries are three operands for each of a bf16 one.  Past 64 channels they stand in LDS, the same for every wave, as the lanes take them,
// [block][half][term][lane]: in registers they leave one wave a SIMD at 128 channels (50 rows on 6007 tokens 65 -> 57 us, 400 on 3000 74.5 -> 67.6), and
// spill at 256 (211 on 6007 202 -> 129).  At 64 they fit, and reading them costs more (211 on 6007, four waves, 46.9 -> 52.0).
template <typename A>
constexpr bool queries_in_lds(int dt) { return sizeof(A) == 4 && dt > 64; }
// Whether two waves a SIMD fit: (queries,) O and a step's operands in 256 registers.
constexpr bool two_a_simd(int dt) { return dt <= 128; }
// per wave O, and m and l per column
constexpr int lds_bytes(int waves, int dt) { return waves * (kCols * dt * 4 + 2 * kCols * 4); }

template <typename A, int DT, bool kExact, int W>
__global__ __launch_bounds__(64 * W, two_a_simd(DT) ? 2 : 1) void prefill_q8_split_kernel(Args x, Deal deal)
{
    constexpr int kTerms = terms_of<A>(), kK = DT / 32, kV = DT / 32;      // 16-byte loads of a lane for a step's keys, and for its values
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const AttnArgs& a = x.a;
    const int hkv = a.c.hkv, hq = a.hq, G = hq / hkv, D = kExact ? DT : a.c.d, ps = a.c.ps, chunks = D >> 4;
    int g, j;
    if (!place_of(deal, hkv, g, j)) return;
    int s = -1, qt = 0, N = 0, P = 0, row0 = 0;
    find_tile<kCols>(a, j, G, s, qt, N, P, row0);
    if (s < 0) return;                              // beyond the batch's tiles
    const int ctx = P + N;
    const int col0 = qt * kCols, cols = min(N * G - col0, kCols);
    const Columns columns(col0, G);
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, hi = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = min(n, cols - 1);                                         // columns beyond the tile repeat the last one
    const int token = columns.token(col), head = columns.head(col, token), qpos = P + token;
    const int64_t row = ((int64_t)row0 + token) * hq + (int64_t)g * G + head;
    const int steps = (P + columns.token(cols - 1)) / kTok + 1;               // of the workgroup
    const int per = (steps + W - 1) / W, u0 = w * per, my_n = max(0, min(per, steps - u0));
    const int first_masked = (P + columns.token(0) + 1) / kTok;               // first step holding a key that the first column may not see

    float m = -INFINITY, lsum = 0.f;
    f32x16 o[kV];
#pragma unroll
    for (int mb = 0; mb < kV; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[mb][i] = 0.f;

    // columns' queries as B operands: k-step (i, half) covers channels (2 i + hi) * 16 + half * 8 .. + 7
    auto query = [&](int i, int half, bf16x8 (&q)[kTerms]) {
        const int chunk = 2 * i + hi;
        if (kExact || chunk < chunks) to_terms((const A*)a.q + row * D + chunk * 16 + half * 8, q);
        else no_terms(q);
    };
    if constexpr (queries_in_lds<A>(DT)) {
        for (int i = w; i < 2 * kK; i += W) {
            bf16x8 q[kTerms];
            query(i >> 1, i & 1, q);
#pragma unroll
            for (int t = 0; t < kTerms; ++t) *reinterpret_cast<bf16x8*>(lds + (i * kTerms + t) * 1024 + lane * 16) = q[t];
        }
        __syncthreads();
    }
    if (my_n > 0) {
        typedef const __attribute__((address_space(4))) int32_t* cptr_t;
        const cptr_t bt = (cptr_t)(uintptr_t)(a.bt + (int64_t)s * a.max_pages);
        const int last_grp = (ctx - 1) >> 4, gshift = a.c.ps_shift - 4, gmask = (1 << gshift) - 1;
        const int kg = (n >> 2) & 1;                                          // this lane's group of the keys
        bf16x8 q[queries_in_lds<A>(DT) ? 1 : kK][2][kTerms];
        if constexpr (!queries_in_lds<A>(DT)) {
#pragma unroll
            for (int i = 0; i < kK; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) query(i, half, q[i][half]);
        }
        u32x4 k[kK], v[kV], ve;
        uint32_t ke;
        const uint32_t k_off = (uint32_t)((n >> 3) * chunks * 64 + (n & 3) * 16), ke_off = (uint32_t)((n & 3) * 4 + (n >> 3));
        const Finder find(a.c, D, g);
        struct Ids { int a, b; };                                             // pages of a step's two groups, fetched a step before they are used
        auto ids_of = [&](int st) {
            const int grp = 2 * (u0 + st);
            return Ids{bt[min(grp, last_grp) >> gshift], bt[min(grp + 1, last_grp) >> gshift]};
        };
        struct Places { Where a, b; };
        auto places_of = [&](int st, Ids id) {
            const int grp = 2 * (u0 + st);
            return Places{find.at(id.a, min(grp, last_grp) & gmask), find.at(id.b, min(grp + 1, last_grp) & gmask)};
        };
        auto load_k = [&](const Places& p) {
            const uint8_t* kp = data_at(a.c.k, kg ? p.b.data : p.a.data) + k_off;
#pragma unroll
            for (int i = 0; i < kK; ++i) {
                const int chunk = kExact ? 2 * i + hi : min(2 * i + hi, chunks - 1);     // (beyond: times zeros of the query)
                k[i] = *reinterpret_cast<const u32x4*>(kp + chunk * 64);
            }
            ke = exps_at(x.exps, kg ? p.b.exps : p.a.exps)[ke_off];
        };
        auto load_v = [&](const Places& p) {
            const uint8_t* vp = data_at(a.c.v, hi ? p.b.data : p.a.data);
#pragma unroll
            for (int mb = 0; mb < kV; ++mb) v[mb] = *reinterpret_cast<const u32x4*>(vp + (kExact ? mb * 32 + n : min(mb * 32 + n, D - 1)) * 16);
            ve = *reinterpret_cast<const u32x4*>(exps_at(x.exps, hi ? p.b.exps : p.a.exps) + ps);
        };
        const float sl2 = a.scale * kLog2e;
        bool noted = false;                                                   // uniform
        Ids ids = ids_of(0);
        Places at = places_of(0, ids);
        load_k(at);
        load_v(at);
        ids = ids_of(1);
        __builtin_amdgcn_sched_barrier(0);
        // (past the wave's last step the requests run on: clamped to the context, never used)
#pragma unroll 1
        for (int st = 0; st < my_n; ++st) {
            f32x16 sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.f;
            const float scale = power(ke);
#pragma unroll
            for (int i = 0; i < kK; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    bf16x8(&qh)[kTerms] = q[queries_in_lds<A>(DT) ? 0 : i][half];
                    if constexpr (queries_in_lds<A>(DT)) {
#pragma unroll
                        for (int t = 0; t < kTerms; ++t) qh[t] = *reinterpret_cast<const bf16x8*>(lds + ((2 * i + half) * kTerms + t) * 1024 + lane * 16);
                    }
                    sc = product(widen8(k[i][2 * half], k[i][2 * half + 1], scale), qh, sc);
                }
            __builtin_amdgcn_sched_barrier(0);
            at = places_of(st + 1, ids);
            load_k(at);
            __builtin_amdgcn_sched_barrier(0);
            // sc[i]: slot i of group hi
            const int tok0 = (u0 + st) * kTok + hi * 16;
            if (u0 + st >= first_masked) {
                asm volatile("");                            // (a branch)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = tok0 + i <= qpos ? sc[i] : -INFINITY;
                // slots behind the last token may hold anything, NaN included: zeros
#pragma unroll
                for (int mb = 0; mb < kV; ++mb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[mb][i] = keep_bytes(v[mb][i], ctx - tok0 - 4 * i);
                noted |= take_nan_out(v);                    // (nan_to_those_that_see_it())
            }
            float mx = sc[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
            mx *= sl2;                                       // scale > 0: max and scaling commute
            // m is shared by the two lanes of a column: if either lane's own maximum outgrew it, combine them
            if (__builtin_amdgcn_ballot_w64(mx > m + kSlack) != 0) {
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m, mx);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
                lsum *= alpha;
#pragma unroll
                for (int mb = 0; mb < kV; ++mb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[mb][i] *= alpha;
                m = m_new;
            }
            const float m_ref = m == -INFINITY ? 0.f : m;
            float psum = 0.f;
            bf16x8 wt[2][kTerms];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(sc[half * 8 + i], sl2, -m_ref));
                psum = add_weights<kTerms>(psum, p);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = times_power(p[i], ve, half * 8 + i);
                to_terms(p, wt[half]);
            }
            lsum += psum;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int mb = 0; mb < kV; ++mb) o[mb] = product(widen8(v[mb][2 * half], v[mb][2 * half + 1], 1.f), wt[half], o[mb]);
            __builtin_amdgcn_sched_barrier(0);
            load_v(at);
            ids = ids_of(st + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (noted) {
            const int last = min((u0 + my_n) * kTok - 1, P + columns.token(cols - 1));
            nan_to_those_that_see_it<kV>(a, find, s, max(u0, first_masked) * kTok, last, qpos, hi, o);
        }
    }
    lsum += __shfl_xor(lsum, 32);

    if constexpr (queries_in_lds<A>(DT)) __syncthreads();                       // (no wave reads its queries any more)
    // the waves' sums, lane by lane: O as quads of channels [wave][quad][lane], then m and l [wave][column]
    f32x4* const part = reinterpret_cast<f32x4*>(lds);
    float* const s_m = reinterpret_cast<float*>(lds + W * kCols * DT * 4);
    float* const s_l = s_m + W * kCols;
    constexpr int kQuads = DT / 8;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
        const int b = (i & 3) * 4;
        part[(w * kQuads + i) * 64 + lane] = f32x4{o[i >> 2][b], o[i >> 2][b + 1], o[i >> 2][b + 2], o[i >> 2][b + 3]};
    }
    if (hi == 0) { s_m[w * kCols + n] = m; s_l[w * kCols + n] = lsum; }
    __syncthreads();
    float f[W], top = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, s_m[i * kCols + n]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        f[i] = __builtin_amdgcn_exp2f(s_m[i * kCols + n] - ref);              // a wave that saw no key has m = -inf -> 0
        l += f[i] * s_l[i * kCols + n];
    }
    const float inv = 1.0f / l;
    if (n >= cols) return;
    A* const out = (A*)a.out + row * D;
    typedef A quad __attribute__((ext_vector_type(4)));
    for (int i = w; i < kQuads; i += W) {                                     // O^T[channel 8 i + 4 hi + e][column n]
        const int d = i * 8 + hi * 4;
        if (!kExact && d >= D) break;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ww = 0; ww < W; ++ww) {
            const f32x4 y = part[(ww * kQuads + i) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += f[ww] * y[e];
        }
        quad y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (A)(acc[e] * inv);
        *reinterpret_cast<quad*>(out + d) = y;
    }
}

template <typename A, int DT, bool kExact, int W>
ag_status launch(const Args& x, hipStream_t st)
{
    constexpr int lds = lds_bytes(W, DT);
    if constexpr (lds > 64 * 1024) {
        static std::atomic<uint64_t> told{0};
        ag_status e = allow_dynamic_lds((const void*)prefill_q8_split_kernel<A, DT, kExact, W>, lds, told);
        if (e) return e;
    }
    const AttnArgs& a = x.a;
    if (a.c.hkv * tiles_bound(a, kCols) + kDealtPast > most_workgroups(64 * W) || (int64_t)a.total_rows * (a.hq / a.c.hkv) > 0x7fffffff) {
        set_error("too many rows for one launch");
        return AG_ERR_INVALID_ARG;
    }
    const Deal deal = deal_of(a, tiles_bound(a, kCols), std::max(1, stream_cus(st) * (two_a_simd(DT) ? 8 / W : 1) / 8));
    prof_before(st);
    hipLaunchKernelGGL((prefill_q8_split_kernel<A, DT, kExact, W>), dim3((unsigned)workgroups_of(deal)), dim3(64 * W), lds, st, x, deal);
    prof_after(st);
    return hip_check(hipGetLastError(), "prefill launch");
}

// Eight waves a workgroup and one workgroup a CU, or four and two: a chain is half as long, or there is room for twice as many, and on
// short contexts less to start and to add up.  Graph replay, eight -> four, us (workgroups): 211 rows on 6007 tokens (216) 34.6 -> 37.2, x 64 25.7 -> 30.5, fp32
// 65.7 -> 73.8, x 64 43.4 -> 46.0; 400 on 6007 (400) 75 -> 66, 500 rows (504) 13.5 -> 9.7, 16 of 30 on 600 (512) 17.0 -> 12.6, fp32 25.3 -> 20.5, x 64 18.4 -> 13.7; 8 of 30 on 100 (256) 6.6 -> 6.1.
// Of several sessions on long contexts the longest make the launch, and half as many again still gain from eight: 6 of 180..305 rows on 110..6229 at 6 / 2
// heads x 64 (294) 27.7 -> 40, 11 of 27..286 on 472..7169 x 128 (314) 45 -> 66.
bool four_waves(const AttnArgs& a, hipStream_t st)
{
    const int64_t few = a.c.hkv * tiles_bound(a, kCols), cus = stream_cus(st);
    return a.max_ctx <= 256 || 2 * few > (a.batch > 1 && a.max_ctx >= 2000 ? 3 : 2) * cus;
}

template <typename A, int DT, bool kExact>
ag_status launch_waves(const Args& x, hipStream_t st)
{
    if constexpr (two_a_simd(DT)) {
        if (!four_waves(x.a, st)) return launch<A, DT, kExact, 8>(x, st);
    }
    return launch<A, DT, kExact, 4>(x, st);
}

// The least of five widths that holds a head: 211 rows on 6007 tokens x 96 in 128 channels 36.8 us, in 96 32.5; x 192 in 256 63.8, in 192 50.6.
template <typename A>
ag_status launch_typed(const Args& x, hipStream_t st)
{
    const int d = x.a.c.d;
    return d == 64 ? launch_waves<A, 64, true>(x, st) : d < 64 ? launch_waves<A, 64, false>(x, st)
         : d == 96 ? launch_waves<A, 96, true>(x, st) : d < 96 ? launch_waves<A, 96, false>(x, st)
         : d == 128 ? launch_waves<A, 128, true>(x, st) : d < 128 ? launch_waves<A, 128, false>(x, st)
         : d == 192 ? launch_waves<A, 192, true>(x, st) : d < 192 ? launch_waves<A, 192, false>(x, st)
         : d == 256 ? launch_waves<A, 256, true>(x, st) : launch_waves<A, 256, false>(x, st);
}

}  // namespace

ag_status launch_prefill_split(const Args& x, hipStream_t st)
{
    return x.a.c.dtype == AG_BF16 ? launch_typed<__bf16>(x, st) : launch_typed<float>(x, st);
}

}  // namespace q8
}  // namespace ag
