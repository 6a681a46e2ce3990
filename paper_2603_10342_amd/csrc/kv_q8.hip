// Append to the 8-bit KV cache, and the way back (include/ag_q8.h): rows of activations <-> e4m3 numbers with a power of two a
// row, in pages.
//
// Bound by HBM, a row once and its bytes once: T * 2 Hkv * (D * sizeof + D + 1).  One workgroup per (touched 16-token group of a
// session, KV head), as the append of the other caches: a group is what the value pool keeps together, 16 slots of a channel in a
// 16-byte run, so that its transposition stays inside the workgroup (through LDS, 16 bytes a lane on both sides of HBM).
// A lane takes 16 channels of a row; the lanes of a row, 2^k >= D / 16 of them in one wave, find its largest size by k exchanges.
#include <algorithm>

#include "find_session.h"
#include "q8_internal.h"

namespace ag {
namespace q8 {
namespace {

constexpr int kGroup = 16;

struct RowArgs {                // one call
    uint8_t *k_pool, *v_pool, *exps;
    void *k, *v;                // rows [T][Hkv][D]
    const int32_t* bt;
    int max_pages;
    const int32_t *prefix_lens, *new_lens, *cu_new;
    int batch, hkv, d, ps, ps_shift, lanes_log2;       // 2^lanes_log2 >= d / 16 lanes a row
};

struct Group {                  // the tokens of a workgroup
    int n_tok, slot0;           // how many, and the first one's slot in its page
    int64_t row0;               // ... and its row
    int64_t page;
};

// A session has at most as many groups as tokens, and at most N / 16 + 2: both summed over the sessions before.
__device__ __forceinline__ bool find_group(const RowArgs& x, Group& o)
{
    const Session f = find_session(x.new_lens, x.prefix_lens, x.cu_new, x.batch, blockIdx.x, [](int ss, int cu) { return min(cu, (cu >> 4) + 2 * ss); });
    const int last_pos = f.prefix + f.new_len - 1, grp = (f.prefix >> 4) + ((int)blockIdx.x - f.first);
    if (f.new_len <= 0 || grp > last_pos >> 4) return false;         // nobody's item
    const int pos0 = max(f.prefix, grp << 4);
    o.n_tok = min(last_pos, (grp << 4) + 15) - pos0 + 1;
    o.slot0 = pos0 & (x.ps - 1);
    o.row0 = f.row0 + (pos0 - f.prefix);
    o.page = x.bt[(int64_t)f.s * x.max_pages + (pos0 >> x.ps_shift)];
    return true;
}

template <typename A>
struct Row16 { u32x4 w[sizeof(A)]; };           // 16 channels: 32 bytes of bf16, 64 of fp32

__device__ __forceinline__ void channels(const Row16<__bf16>& r, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[2 * i] = __builtin_bit_cast(float, r.w[i >> 2][i & 3] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, r.w[i >> 2][i & 3] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void channels(const Row16<float>& r, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __builtin_bit_cast(f32x4, r.w[i >> 2])[i & 3];
}
__device__ __forceinline__ Row16<__bf16> row_of(const u32x4& q, float scale, __bf16)
{
    Row16<__bf16> r;
    r.w[0] = __builtin_bit_cast(u32x4, widen8(q[0], q[1], scale));
    r.w[1] = __builtin_bit_cast(u32x4, widen8(q[2], q[3], scale));
    return r;
}
__device__ __forceinline__ Row16<float> row_of(const u32x4& q, float scale, float)
{
    Row16<float> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
        r.w[i] = __builtin_bit_cast(u32x4, f32x4{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale});
    }
    return r;
}
// Bytes `at` of 16 words, in their order.
template <class Word>
__device__ __forceinline__ u32x4 gather_bytes(Word word, int at)
{
    const uint32_t two = (uint32_t)at | (uint32_t)(at + 4) << 8 | 0x0C0C0000u;       // one of each of two words
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(word(4 * i + 1), word(4 * i), two), hi = __builtin_amdgcn_perm(word(4 * i + 3), word(4 * i + 2), two);
        r[i] = lo | hi << 16;
    }
    return r;
}

template <typename A>
__global__ __launch_bounds__(256) void append_q8_kernel(RowArgs x)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t s_v[];      // [token][d] e4m3
    Group o;
    if (!find_group(x, o)) return;
    const int tid = threadIdx.x, h = blockIdx.y, d = x.d, chunks = d >> 4;
    uint8_t* const kp = x.k_pool + (o.page * x.hkv + h) * (int64_t)(d * x.ps);
    uint8_t* const vp = x.v_pool + (o.page * x.hkv + h) * (int64_t)(d * x.ps);
    uint8_t* const ep = x.exps + (o.page * x.hkv + h) * (int64_t)(2 * x.ps);
    for (int idx = tid; idx < (2 * o.n_tok) << x.lanes_log2; idx += 256) {             // keys, then values
        const int line = idx >> x.lanes_log2, c = idx & ((1 << x.lanes_log2) - 1);
        const bool value = line >= o.n_tok;
        const int t = value ? line - o.n_tok : line;
        Row16<A> raw = {};
        if (c < chunks) {
            const u32x4* src = reinterpret_cast<const u32x4*>((const A*)(value ? x.v : x.k) + ((o.row0 + t) * x.hkv + h) * d + c * 16);
#pragma unroll
            for (int i = 0; i < (int)sizeof(A); ++i) raw.w[i] = src[i];
        }
        float f[16];
        channels(raw, f);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, size_of(f[i]));
        for (int m = 1; m < 1 << x.lanes_log2; m <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m));
        const uint32_t e = exponent_byte(most);
        u32x4 q;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = quantise4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], e);
        const int slot = o.slot0 + t;
        if (c < chunks) {
            if (value) *reinterpret_cast<u32x4*>(s_v + t * d + c * 16) = q;
            else *reinterpret_cast<u32x4*>(kp + ((slot >> 2) * chunks + c) * 64 + (slot & 3) * 16) = q;
        }
        if (c == 0) ep[value ? x.ps + slot : (slot & ~15) + key_place(slot)] = (uint8_t)e;
    }
    __syncthreads();
    uint8_t* const vg = vp + (o.slot0 >> 4) * 16 * d;                // [channel][16 slots]
    if (o.n_tok == kGroup) {
        for (int ch = tid; ch < d; ch += 256)
            *reinterpret_cast<u32x4*>(vg + ch * 16) = gather_bytes([&](int t) { return *reinterpret_cast<const uint32_t*>(s_v + t * d + (ch & ~3)); }, ch & 3);
    } else {                                                         // the other slots' bytes stay as they are
        for (int idx = tid; idx < o.n_tok * d; idx += 256) {
            const int t = idx / d, ch = idx - t * d;
            vg[ch * 16 + (o.slot0 & 15) + t] = s_v[idx];
        }
    }
}

template <typename A>
__global__ __launch_bounds__(256) void read_q8_kernel(RowArgs x)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t s_v[];      // [chunk of 16 channels][channel][16 slots], chunks 16 bytes apart
    constexpr int kChunk = 16 * 16 + 16;
    Group o;
    if (!find_group(x, o)) return;
    const int tid = threadIdx.x, h = blockIdx.y, d = x.d, chunks = d >> 4;
    const uint8_t* const kp = x.k_pool + (o.page * x.hkv + h) * (int64_t)(d * x.ps);
    const uint8_t* const vg = x.v_pool + (o.page * x.hkv + h) * (int64_t)(d * x.ps) + (o.slot0 >> 4) * 16 * d;
    const uint8_t* const ep = x.exps + (o.page * x.hkv + h) * (int64_t)(2 * x.ps);
    for (int ch = tid; ch < d; ch += 256)
        *reinterpret_cast<u32x4*>(s_v + (ch >> 4) * kChunk + (ch & 15) * 16) = *reinterpret_cast<const u32x4*>(vg + ch * 16);
    __syncthreads();
    for (int idx = tid; idx < 2 * o.n_tok * chunks; idx += 256) {      // keys, then values
        const int line = idx / chunks, c = idx - line * chunks;
        const bool value = line >= o.n_tok;
        const int t = value ? line - o.n_tok : line, slot = o.slot0 + t;
        u32x4 q;
        if (value) {
            const uint8_t* at = s_v + c * kChunk + (slot & 12);
            q = gather_bytes([&](int i) { return *reinterpret_cast<const uint32_t*>(at + i * 16); }, slot & 3);
        } else {
            q = *reinterpret_cast<const u32x4*>(kp + ((slot >> 2) * chunks + c) * 64 + (slot & 3) * 16);
        }
        const Row16<A> r = row_of(q, power(ep[value ? x.ps + slot : (slot & ~15) + key_place(slot)]), A(0));
        u32x4* dst = reinterpret_cast<u32x4*>((A*)(value ? x.v : x.k) + ((o.row0 + t) * x.hkv + h) * d + c * 16);
#pragma unroll
        for (int i = 0; i < (int)sizeof(A); ++i) dst[i] = r.w[i];
    }
}

// every session touches at most N_s / 16 + 2 groups, and every group has a token
ag_status grid_of(const CacheView& c, int batch, int total, dim3* grid)
{
    const int64_t items = std::min<int64_t>(total / 16 + 2 * (int64_t)batch, total);
    if (items > 0x7fffffff || c.hkv > 65535) { set_error("too many groups or heads for one launch"); return AG_ERR_INVALID_ARG; }
    *grid = dim3((unsigned)items, c.hkv);
    return AG_OK;
}

int lanes_log2(int chunks)
{
    int k = 0;
    while ((1 << k) < chunks) ++k;
    return k;
}

}  // namespace

ag_status launch_append(const CacheView& c, uint8_t* exps, const void* k_new, const void* v_new, const int32_t* bt, int max_pages,
                        const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st)
{
    dim3 grid;
    ag_status e = grid_of(c, batch, total_new, &grid);
    if (e) return e;
    const RowArgs x = {(uint8_t*)c.k, (uint8_t*)c.v, exps, (void*)k_new, (void*)v_new, bt, max_pages, prefix_lens, new_lens, cu_new,
                       batch, c.hkv, c.d, c.ps, c.ps_shift, lanes_log2(c.d / 16)};
    if (c.dtype == AG_BF16) hipLaunchKernelGGL(append_q8_kernel<__bf16>, grid, dim3(256), kGroup * c.d, st, x);
    else hipLaunchKernelGGL(append_q8_kernel<float>, grid, dim3(256), kGroup * c.d, st, x);
    return hip_check(hipGetLastError(), "append launch");
}

ag_status launch_read(const CacheView& c, const uint8_t* exps, void* k_out, void* v_out, const int32_t* bt, int max_pages,
                      const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st)
{
    dim3 grid;
    ag_status e = grid_of(c, batch, total_new, &grid);
    if (e) return e;
    const RowArgs x = {(uint8_t*)c.k, (uint8_t*)c.v, (uint8_t*)exps, k_out, v_out, bt, max_pages, prefix_lens, new_lens, cu_new,
                       batch, c.hkv, c.d, c.ps, c.ps_shift, lanes_log2(c.d / 16)};
    const int lds = c.d / 16 * (16 * 16 + 16);
    if (c.dtype == AG_BF16) hipLaunchKernelGGL(read_q8_kernel<__bf16>, grid, dim3(256), lds, st, x);
    else hipLaunchKernelGGL(read_q8_kernel<float>, grid, dim3(256), lds, st, x);
    return hip_check(hipGetLastError(), "read launch");
}

}  // namespace q8
}  // namespace ag
