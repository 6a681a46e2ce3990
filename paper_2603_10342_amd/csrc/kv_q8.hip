// Append to the 8-bit KV cache, and the way back (include/ag_q8.h): rows of activations <-> e4m3 numbers with a power of two a
// row, in pages.
//
// Bound by HBM, a row once and its bytes once: T * 2 Hkv * (D * sizeof + D + 1).  One workgroup per touched 16-token group of a
// session and KV head, or several heads (grid_of()): a group is what the value pool keeps together, 16 slots of a channel in a
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

// kHeads KV heads a workgroup: their rows of a token lie side by side.
template <typename A, int kHeads>
__global__ __launch_bounds__(256) void append_q8_kernel(RowArgs x)
{
    constexpr int kAtOnce = kHeads == 1 ? 1 : 2;
    extern __shared__ __attribute__((aligned(16))) uint8_t s_v[];      // [head][token][d] e4m3
    Group o;
    if (!find_group(x, o)) return;
    const int tid = threadIdx.x, h0 = blockIdx.y * kHeads, d = x.d, chunks = d >> 4, ll = x.lanes_log2;
    const int64_t block = (int64_t)d * x.ps, at = o.page * x.hkv + h0;
    const int lines = 2 * o.n_tok * kHeads;                            // rows: keys of the tokens, then values; the heads of a token in turn
    for (int i0 = tid; i0 < lines << ll; i0 += 256 * kAtOnce) {
        Row16<A> raw[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int idx = i0 + j * 256, line = idx >> ll, c = idx & ((1 << ll) - 1), tt = line / kHeads, t = tt >= o.n_tok ? tt - o.n_tok : tt;
            raw[j] = {};
            if (line < lines && c < chunks) {
                const u32x4* src = reinterpret_cast<const u32x4*>((const A*)(tt >= o.n_tok ? x.v : x.k) + ((o.row0 + t) * x.hkv + h0 + line % kHeads) * d + c * 16);
#pragma unroll
                for (int i = 0; i < (int)sizeof(A); ++i) raw[j].w[i] = src[i];
            }
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int idx = i0 + j * 256, line = idx >> ll, c = idx & ((1 << ll) - 1), tt = line / kHeads, hh = line % kHeads;
            if (line >= lines) break;                                  // (a row's lanes alike)
            const bool value = tt >= o.n_tok;
            const int t = value ? tt - o.n_tok : tt, slot = o.slot0 + t;
            float f[16];
            channels(raw[j], f);
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) most = max(most, size_of(f[i]));
            for (int m = 1; m < 1 << ll; m <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m));
            const uint32_t e = exponent_byte(most);
            u32x4 q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = quantise4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3], e);
            if (c < chunks) {
                if (value) *reinterpret_cast<u32x4*>(s_v + (hh * kGroup + t) * d + c * 16) = q;
                else *reinterpret_cast<u32x4*>(x.k_pool + (at + hh) * block + ((slot >> 2) * chunks + c) * 64 + (slot & 3) * 16) = q;
            }
            if (c == 0) x.exps[(at + hh) * (2 * x.ps) + (value ? x.ps + slot : (slot & ~15) + key_place(slot))] = (uint8_t)e;
        }
    }
    __syncthreads();
    uint8_t* const vg = x.v_pool + at * block + (o.slot0 >> 4) * 16 * d;              // [channel][16 slots]
    if (o.n_tok == kGroup) {
        for (int i = tid; i < kHeads * d; i += 256) {
            const int hh = kHeads == 1 ? 0 : i / d, ch = i - hh * d;
            const uint8_t* src = s_v + hh * kGroup * d + (ch & ~3);
            *reinterpret_cast<u32x4*>(vg + hh * block + ch * 16) = gather_bytes([&](int t) { return *reinterpret_cast<const uint32_t*>(src + t * d); }, ch & 3);
        }
    } else {                                                         // the other slots' bytes stay as they are
        for (int i = tid; i < kHeads * o.n_tok * d; i += 256) {
            const int line = i / d, ch = i - line * d, hh = kHeads == 1 ? 0 : line / o.n_tok, t = line - hh * o.n_tok;
            vg[hh * block + ch * 16 + (o.slot0 & 15) + t] = s_v[(hh * kGroup + t) * d + ch];
        }
    }
}

template <typename A, int kHeads>
__global__ __launch_bounds__(256) void read_q8_kernel(RowArgs x)
{
    constexpr int kAtOnce = kHeads == 1 ? 1 : 2;
    extern __shared__ __attribute__((aligned(16))) uint8_t s_v[];      // [head][chunk of 16 channels][channel][16 slots], chunks 16 bytes apart
    constexpr int kChunk = 16 * 16 + 16;
    Group o;
    if (!find_group(x, o)) return;
    const int tid = threadIdx.x, h0 = blockIdx.y * kHeads, d = x.d, chunks = d >> 4;
    const int64_t block = (int64_t)d * x.ps, at = o.page * x.hkv + h0;
    const uint8_t* const vg = x.v_pool + at * block + (o.slot0 >> 4) * 16 * d;
    for (int i = tid; i < kHeads * d; i += 256) {
        const int hh = kHeads == 1 ? 0 : i / d, ch = i - hh * d;
        *reinterpret_cast<u32x4*>(s_v + (hh * chunks + (ch >> 4)) * kChunk + (ch & 15) * 16) = *reinterpret_cast<const u32x4*>(vg + hh * block + ch * 16);
    }
    __syncthreads();
    const int lines = 2 * o.n_tok * kHeads;                            // rows: keys of the tokens, then values; the heads of a token in turn
    for (int i0 = tid; i0 < lines * chunks; i0 += 256 * kAtOnce) {
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int idx = i0 + j * 256, line = idx / chunks, c = idx - line * chunks, tt = line / kHeads, hh = line % kHeads;
            if (line >= lines) break;
            const bool value = tt >= o.n_tok;
            const int t = value ? tt - o.n_tok : tt, slot = o.slot0 + t;
            u32x4 q;
            if (value) {
                const uint8_t* src = s_v + (hh * chunks + c) * kChunk + (slot & 12);
                q = gather_bytes([&](int i) { return *reinterpret_cast<const uint32_t*>(src + i * 16); }, slot & 3);
            } else {
                q = *reinterpret_cast<const u32x4*>(x.k_pool + (at + hh) * block + ((slot >> 2) * chunks + c) * 64 + (slot & 3) * 16);
            }
            const uint32_t e = x.exps[(at + hh) * (2 * x.ps) + (value ? x.ps + slot : (slot & ~15) + key_place(slot))];
            const Row16<A> r = row_of(q, power(e), A(0));
            u32x4* dst = reinterpret_cast<u32x4*>((A*)(value ? x.v : x.k) + ((o.row0 + t) * x.hkv + h0 + hh) * d + c * 16);
#pragma unroll
            for (int i = 0; i < (int)sizeof(A); ++i) dst[i] = r.w[i];
        }
    }
}

// every session touches at most N_s / 16 + 2 groups, and every group has a token
ag_status grid_of(const CacheView& c, int batch, int total, dim3* grid, int* heads)
{
    const int64_t items = std::min<int64_t>(total / 16 + 2 * (int64_t)batch, total);
    if (items > most_workgroups(256) || c.hkv > 65535) { set_error("too many groups or heads for one launch"); return AG_ERR_INVALID_ARG; }
    // KV heads a workgroup takes.  A group of one is the least latency, but the chip starts a workgroup every 2 ns: past 8192 of them several
    // heads together, up to 256 channels.  1, 2, 4 heads, us, 8 KV heads: 100 sessions of 1000..2000 tokens append x 64 156, 109, 93,
    // x 128 213, 182, 183, x 256 424, 416, 459, fp32 x 128 303, 301, 319; read x 64 172, 117, 93, x 128 254, 188, 194, x 256 385, 389, 437; but 32 of
    // 100..300 append x 128 10.4, 13.1, 14.7, 64 of 2..20 6.0, 8.8, 11.2.
    *heads = 1;
    if (items * c.hkv > 8192)
        while (*heads < 4 && c.hkv % (2 * *heads) == 0 && 2 * *heads * c.d <= 256) *heads *= 2;
    *grid = dim3((unsigned)items, c.hkv / *heads);
    return AG_OK;
}

int lanes_log2(int chunks)
{
    int k = 0;
    while ((1 << k) < chunks) ++k;
    return k;
}

template <typename A>
void append_heads(int heads, dim3 grid, int lds, hipStream_t st, const RowArgs& x)
{
    if (heads == 4) hipLaunchKernelGGL((append_q8_kernel<A, 4>), grid, dim3(256), lds, st, x);
    else if (heads == 2) hipLaunchKernelGGL((append_q8_kernel<A, 2>), grid, dim3(256), lds, st, x);
    else hipLaunchKernelGGL((append_q8_kernel<A, 1>), grid, dim3(256), lds, st, x);
}
template <typename A>
void read_heads(int heads, dim3 grid, int lds, hipStream_t st, const RowArgs& x)
{
    if (heads == 4) hipLaunchKernelGGL((read_q8_kernel<A, 4>), grid, dim3(256), lds, st, x);
    else if (heads == 2) hipLaunchKernelGGL((read_q8_kernel<A, 2>), grid, dim3(256), lds, st, x);
    else hipLaunchKernelGGL((read_q8_kernel<A, 1>), grid, dim3(256), lds, st, x);
}

}  // namespace

ag_status launch_append(const CacheView& c, uint8_t* exps, const void* k_new, const void* v_new, const int32_t* bt, int max_pages,
                        const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st)
{
    dim3 grid;
    int heads;
    ag_status e = grid_of(c, batch, total_new, &grid, &heads);
    if (e) return e;
    const RowArgs x = {(uint8_t*)c.k, (uint8_t*)c.v, exps, (void*)k_new, (void*)v_new, bt, max_pages, prefix_lens, new_lens, cu_new,
                       batch, c.hkv, c.d, c.ps, c.ps_shift, lanes_log2(c.d / 16)};
    const int lds = heads * kGroup * c.d;
    if (c.dtype == AG_BF16) append_heads<__bf16>(heads, grid, lds, st, x);
    else append_heads<float>(heads, grid, lds, st, x);
    return hip_check(hipGetLastError(), "append launch");
}

ag_status launch_read(const CacheView& c, const uint8_t* exps, void* k_out, void* v_out, const int32_t* bt, int max_pages,
                      const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st)
{
    dim3 grid;
    int heads;
    ag_status e = grid_of(c, batch, total_new, &grid, &heads);
    if (e) return e;
    const RowArgs x = {(uint8_t*)c.k, (uint8_t*)c.v, (uint8_t*)exps, k_out, v_out, bt, max_pages, prefix_lens, new_lens, cu_new,
                       batch, c.hkv, c.d, c.ps, c.ps_shift, lanes_log2(c.d / 16)};
    const int lds = heads * (c.d / 16) * (16 * 16 + 16);
    if (c.dtype == AG_BF16) read_heads<__bf16>(heads, grid, lds, st, x);
    else read_heads<float>(heads, grid, lds, st, x);
    return hip_check(hipGetLastError(), "read launch");
}

}  // namespace q8
}  // namespace ag
