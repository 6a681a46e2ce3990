// Rotary positions (include/ag_rope.h): rows rotated by their position, and the append that rotates keys and queries on the way.
//
//     a' = m (a cos - b sin)      b' = m (b cos + a sin)      at the angle 2 pi p turns[i] of pair i
//
// Bound by HBM, every row read once and written once: 2 T H D sizeof, and T (2 Hq + 4 Hkv) D sizeof for the append.  A cosine and a sine are about
// twenty 64-bit operations, so that a workgroup finds those of its tokens once, in LDS, while its first rows are on their way, and all heads take them from
// there.  A lane holds eight whole pairs, two 16-byte runs of bf16: both layouts work on registers alone.
#include <algorithm>

#include "find_session.h"
#include "rope_internal.h"

namespace ag {
namespace rope {
namespace {

constexpr int kMostPairs = 128;

// kTok consecutive tokens a workgroup.
template <typename A, bool kPairs, int kTok>
__global__ __launch_bounds__(256) void rope_rows_kernel(RowsArgs x)
{
    constexpr int kAtOnce = kTok == 1 ? 1 : 4;
    __shared__ f32x2 s_cs[kTok][kMostPairs];
    __shared__ int s_valid[kTok];
    const Units us(x.d, x.r.half);
    const int tid = threadIdx.x, t0 = blockIdx.x * kTok, per = us.count(), per_token = x.heads * per;
    const int n = min(kTok, x.total - t0) * per_token;
    const A* const src = (const A*)x.x;
    A* const dst = (A*)x.y;
    const bool in_place = x.x == x.y;
    struct Place { int token, head, u; };
    auto place = [&](int idx) {
        const int row = idx / per, t = kTok == 1 ? 0 : row / x.heads;
        return Place{t, row - t * x.heads, idx - row * per};
    };
    Unit<A> r[kAtOnce];
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int idx = i0 + j * 256;
            if (idx >= n) break;
            const Place p = place(idx);
            load_unit<kPairs>(us, src + (int64_t)(t0 + p.token) * x.xt + (int64_t)p.head * x.xh, p.u, r[j]);
        }
    };
    load(tid);
    const int w = tid >> 6, lane = tid & 63;
    if (w < kTok) {                                                    // a wave finds its token
        const int t = t0 + w;
        const Session f = find_session(x.new_lens, x.prefix_lens, x.cu_new, x.batch, t, [](int, int cu) { return cu; });
        const bool valid = t < x.total && t - f.row0 < f.new_len;
        if (valid)
            for (int i = lane; i < x.r.half; i += 64) s_cs[w][i] = cos_sin(f.prefix + (t - f.row0), x.r, i);
        if (lane == 0) s_valid[w] = valid;
    }
    __syncthreads();
    for (int i0 = tid;;) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int idx = i0 + j * 256;
            if (idx >= n) break;
            const Place p = place(idx);
            if (!s_valid[p.token] || (in_place && p.u >= us.rotated)) continue;
            turn_unit<kPairs>(us, p.u, s_cs[p.token], r[j]);
            store_unit<kPairs>(us, dst + (int64_t)(t0 + p.token) * x.yt + (int64_t)p.head * x.yh, p.u, r[j]);
        }
        i0 += 256 * kAtOnce;
        if (i0 >= n) break;
        load(i0);
    }
}

// One workgroup per touched 16-token group of a session and KV head: its keys and values, and the group's query heads.  Keys and values go
// through LDS, from rows that are read whole to runs of slots that are written whole.
// kStream: what is written is more than the last cache holds, and marked so that it does not go through the nearer ones (8 x 4096 tokens, 32 and 8 heads x 128, 403 MB
// written: 186 -> 172 us of 805 MB; a step's tokens are read next, and cost 5.0 -> 5.2 us so).
constexpr int kGroup = 16;

template <typename A, bool kPairs, bool kStream>
__global__ __launch_bounds__(256) void append_rope_kernel(AppendArgs x)
{
    constexpr int kAtOnce = 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int d = x.c.d, chunks = d >> 3, hkv = x.c.hkv, h = blockIdx.y, tid = threadIdx.x, ps = x.c.ps;
    const int pitch = d + 16 / (int)sizeof(A);                         // 16 bytes more than a row: the slots of a chunk lie in different banks
    A* const s_k = reinterpret_cast<A*>(smem);                         // [token][pitch]
    A* const s_v = s_k + kGroup * pitch;
    f32x2* const s_cs = reinterpret_cast<f32x2*>(s_v + kGroup * pitch);

    // a session has at most as many groups as tokens, and at most N / 16 + 2: both summed over the sessions before
    const Session f = find_session(x.new_lens, x.prefix_lens, x.cu_new, x.batch, blockIdx.x, [](int ss, int cu) { return min(cu, (cu >> 4) + 2 * ss); });
    const int last_pos = f.prefix + f.new_len - 1, grp = (f.prefix >> 4) + ((int)blockIdx.x - f.first);
    if (f.new_len <= 0 || grp > last_pos >> 4) return;                 // nobody's item
    const int pos0 = max(f.prefix, grp << 4), n_tok = min(last_pos, (grp << 4) + 15) - pos0 + 1;
    const int64_t row0 = f.row0 + (pos0 - f.prefix);
    const int64_t page = x.bt[(int64_t)f.s * x.max_pages + (pos0 >> x.c.ps_shift)];
    const int slot0 = pos0 & (ps - 1);

    const Units us(d, x.r.half);
    const int per = us.count(), G = x.q ? x.hq / hkv : 0, nk = n_tok * per, nv = n_tok * chunks, nq = n_tok * G * per;
    Unit<A> rk, rq[kAtOnce];
    auto load_k = [&](int i) {
        const int t = i / per;
        if (i < nk) load_unit<kPairs>(us, (const A*)x.k_new + ((row0 + t) * hkv + h) * d, i - t * per, rk);
    };
    auto q_row = [&](int i, int& t, int& u) {                          // row of q that unit i belongs to
        const int row = i / per;
        t = row / G;
        u = i - row * per;
        return ((row0 + t) * x.hq + h * G + (row - t * G)) * d;
    };
    auto load_q = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = i0 + j * 256;
            if (i >= nq) break;
            int t, u;
            const int64_t row = q_row(i, t, u);
            load_unit<kPairs>(us, (const A*)x.q + row, u, rq[j]);
        }
    };
    load_k(tid);
    load_q(tid);
    for (int i = tid; i < nv; i += 256) {
        const int t = i / chunks, c = i - t * chunks;
        *reinterpret_cast<Eight<A>*>(s_v + t * pitch + c * 8) = *reinterpret_cast<const Eight<A>*>((const A*)x.v_new + ((row0 + t) * hkv + h) * d + c * 8);
    }
    for (int i = tid; i < n_tok * x.r.half; i += 256) {
        const int t = i / x.r.half;
        s_cs[i] = cos_sin(pos0 + t, x.r, i - t * x.r.half);
    }
    __syncthreads();
    for (int i = tid; i < nk;) {
        const int t = i / per, u = i - t * per;
        turn_unit<kPairs>(us, u, s_cs + t * x.r.half, rk);
        store_unit<kPairs>(us, s_k + t * pitch, u, rk);
        i += 256;
        load_k(i);
    }
    for (int i0 = tid; i0 < nq;) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = i0 + j * 256;
            if (i >= nq) break;
            int t, u;
            const int64_t row = q_row(i, t, u);
            turn_unit<kPairs>(us, u, s_cs + t * x.r.half, rq[j]);
            store_unit<kPairs, kStream>(us, (A*)x.q_out + row, u, rq[j]);
        }
        i0 += 256 * kAtOnce;
        load_q(i0);
    }
    __syncthreads();

    const int64_t block = (page * hkv + h) * (int64_t)d * ps;
    A *const kpage = (A*)x.c.k + block, *const vpage = (A*)x.c.v + block;
    for (int i = tid; i < nv; i += 256) {                              // keys: neighbouring lanes, neighbouring slots
        const int c = i / n_tok, t = i - c * n_tok;
        store_eight<kStream>(kpage + ((int64_t)c * ps + slot0 + t) * 8, *reinterpret_cast<const Eight<A>*>(s_k + t * pitch + c * 8));
    }
    if (n_tok == kGroup) {                                             // values of a whole group: chunks of eight slots
        for (int i = tid; i < 2 * d; i += 256) {
            const int half = i >= d, ch = i - half * d;
            struct alignas(16) { A e[8]; } v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v.e[e] = s_v[(half * 4 + e) * pitch + ch];
                v.e[4 + e] = s_v[(8 + half * 4 + e) * pitch + ch];
            }
            store_eight<kStream>(vpage + ((int64_t)((slot0 >> 3) + half) * d + ch) * 8, __builtin_bit_cast(Eight<A>, v));
        }
    } else {                                                           // the other slots stay as they are
        for (int i = tid; i < n_tok * d; i += 256) {
            const int ch = i / n_tok, t = i - ch * n_tok;
            vpage[v_offset(slot0 + t, ch, ps, d)] = s_v[t * pitch + ch];
        }
    }
}

template <typename A, bool kPairs>
ag_status rows_typed(const RowsArgs& a, hipStream_t st)
{
    // Tokens a workgroup: one while the chip holds them all at once, four beyond, whose loads then keep memory busy.  32 heads of 128 channels, us, one / four:
    // 128 tokens 4.2 / 5.1, 2048 6.5 / 8.1, 4096 13.1 / 13.0, 8192 21.6 / 21.3
    constexpr int kMany = 2048;
    if (a.total <= kMany) hipLaunchKernelGGL((rope_rows_kernel<A, kPairs, 1>), dim3(a.total), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((rope_rows_kernel<A, kPairs, 4>), dim3((a.total + 3) / 4), dim3(256), 0, st, a);
    return hip_check(hipGetLastError(), "rope launch");
}

template <typename A, bool kPairs>
void append_typed(const AppendArgs& a, dim3 grid, size_t lds, hipStream_t st)
{
    // What the chip's 256 MB cache cannot keep anyway is written with the streaming hint; what fits stays for the attention that reads it.  32768 tokens, 32 + 8 heads of
    // 128: 173 us with, 186 without; 4096 tokens and the prefill of them 58.3 with, 56.9 without (the append alone 18.9 and 20.8)
    const int64_t written = (int64_t)a.total * (2 * a.c.hkv + a.hq) * a.c.d * (int64_t)sizeof(A);
    if (written > 256ll << 20) hipLaunchKernelGGL((append_rope_kernel<A, kPairs, true>), grid, dim3(256), lds, st, a);
    else hipLaunchKernelGGL((append_rope_kernel<A, kPairs, false>), grid, dim3(256), lds, st, a);
}

}  // namespace

ag_status launch_rows(const RowsArgs& a, hipStream_t st)
{
    if (a.dtype == AG_BF16) return a.layout == AG_ROPE_PAIRS ? rows_typed<__bf16, true>(a, st) : rows_typed<__bf16, false>(a, st);
    return a.layout == AG_ROPE_PAIRS ? rows_typed<float, true>(a, st) : rows_typed<float, false>(a, st);
}

ag_status launch_append(const AppendArgs& a, hipStream_t st)
{
    // every session touches at most N_s / 16 + 2 groups, and every group has a token
    const int64_t items = std::min<int64_t>(a.total / 16 + 2 * (int64_t)a.batch, a.total);
    const dim3 grid((unsigned)items, a.c.hkv);
    const size_t el = a.c.dtype == AG_BF16 ? 2 : 4;
    const size_t lds = 2 * kGroup * (a.c.d * el + 16) + kGroup * a.r.half * sizeof(f32x2);
    const bool pairs = a.layout == AG_ROPE_PAIRS;
    if (a.c.dtype == AG_BF16) pairs ? append_typed<__bf16, true>(a, grid, lds, st) : append_typed<__bf16, false>(a, grid, lds, st);
    else pairs ? append_typed<float, true>(a, grid, lds, st) : append_typed<float, false>(a, grid, lds, st);
    return hip_check(hipGetLastError(), "append launch");
}

}  // namespace rope
}  // namespace ag
