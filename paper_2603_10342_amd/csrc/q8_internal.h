// Internal declarations of the 8-bit cache (include/ag_q8.h): the host's view of it, the launchers, and the device's way between
// e4m3 numbers and the types that arithmetic runs in.
#pragma once

#include <algorithm>

#include "ag_internal.h"
#include "ag_q8.h"
#include "bf16_terms.h"

namespace ag {
namespace q8 {

// An attention problem over an 8-bit cache: a.c holds the pools and the geometry, with the activations' type as its dtype.
struct Args {
    AttnArgs a;
    const uint8_t* exps;
};

ag_status launch_append(const CacheView& c, uint8_t* exps, const void* k_new, const void* v_new, const int32_t* bt, int max_pages,
                        const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st);
ag_status launch_read(const CacheView& c, const uint8_t* exps, void* k_out, void* v_out, const int32_t* bt, int max_pages,
                      const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, hipStream_t st);
size_t    decode_workspace(int batch, int hq, int d, int max_ctx);
ag_status launch_decode(const Args& x, void* ws, hipStream_t st);
ag_status launch_prefill(const Args& x, hipStream_t st);
// few rows: the keys of 32 columns dealt to the waves of one workgroup
ag_status launch_prefill_split(const Args& x, hipStream_t st);

// Workgroups of a launch: HIP refuses 2^32 threads along a dimension of the grid.
constexpr int64_t most_workgroups(int threads) { return 0xFFFFFFFFll / threads; }

// Tiles of `cols` columns of a KV head: sum_s ceil(N_s G / cols) <= total G / cols + batch, and no session has more than ceil(max_new G / cols).
inline int64_t tiles_bound(const AttnArgs& a, int cols)
{
    const int64_t G = a.hq / a.c.hkv;
    return std::min<int64_t>((int64_t)a.total_rows * G / cols + a.batch, (int64_t)a.batch * ((a.max_new * G + cols - 1) / cols));
}

// Where a key's exponent byte stands in its group of 16 slots: the four that a lane of the score product needs are one word.
__host__ __device__ inline int key_place(int slot) { return (slot & 3) * 4 + ((slot >> 2) & 3); }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kExpLo = -110 + 127, kExpHi = 119 + 127;          // of the stored bytes

// 2^(byte - 127)
__device__ __forceinline__ float power(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// x times the power that byte i of four words stands for, by adding to x's exponent: two instructions where a power takes three.  A byte that
// is nobody's may be any: zero stays zero.
__device__ __forceinline__ float times_power(float x, const u32x4& bytes, int i) { return ldexpf(x, (int)((bytes[i >> 2] >> (8 * (i & 3))) & 0xFFu) - 127); }

// |x| in bits, 0 for what is not finite: sizes compare as integers
__device__ __forceinline__ uint32_t size_of(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}
// The byte of a row whose largest size has these bits: 448 is 1.75 * 2^8, so a mantissa above 0.75 takes the next power.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t most)
{
    return (uint32_t)min(max((int)((most + 0x1FFFFFu) >> 23) - 8, kExpLo), kExpHi);
}
// Four numbers as e4m3 under the row's power.  Only the largest power leaves numbers past 448 (they are cut to it); infinities become NaN.
__device__ __forceinline__ uint32_t quantise4(float a, float b, float c, float d, uint32_t byte)
{
    const float inv = power(254 - byte);
    float y[4] = {a * inv, b * inv, c * inv, d * inv};
    if (byte == (uint32_t)kExpHi) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fabsf(y[i]) < INFINITY ? fminf(fmaxf(y[i], -448.f), 448.f) : y[i];
    }
    uint32_t w = 0;
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], (int)w, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], (int)w, true);
}

// Eight e4m3 numbers times a power of two as bf16: exact, four instructions (as fast as an addition: 4 cycles a wave).
__device__ __forceinline__ bf16x8 widen8(uint32_t w0, uint32_t w1, float scale)
{
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
    return __builtin_bit_cast(bf16x8, r);
}
// Two numbers of a word, each times a power of its own, as bf16: exact
template <bool kHigh>
__device__ __forceinline__ uint32_t widen_pair(uint32_t w, float s0, float s1)
{
    const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, kHigh);
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(x[0] * s0), (__bf16)(x[1] * s1)});
}

// Keeps the first `keep` bytes of a word (any `keep`), zeroes the others.
__device__ __forceinline__ uint32_t keep_bytes(uint32_t w, int keep)
{
    return keep >= 4 ? w : keep <= 0 ? 0u : w & ((1u << (8 * keep)) - 1u);
}

// NaN has the largest byte of either sign.  Whether one of the wave's words has one - then those bytes become zeros.
template <int N>
__device__ __forceinline__ bool take_nan_out(u32x4 (&x)[N])
{
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) any |= (x[i][k] & 0x7F7F7F7Fu) + 0x01010101u;          // (no byte carries)
    if (__builtin_amdgcn_ballot_w64((any & 0x80808080u) != 0) == 0) return false;
    asm volatile("");                                                                      // (a branch)
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t nan = ((x[i][k] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
            x[i][k] &= ~((nan << 1) - (nan >> 7));
        }
    return true;
}

// Numbers of the activations' type, exactly, and softmax weights as bf16 terms: operands of the products.  One term of a weight rounds it.
template <typename A>
constexpr int terms_of() { return sizeof(A) == 4 ? 3 : 1; }
__device__ __forceinline__ void as_terms(const Terms& x, bf16x8 (&t)[3])
{
    t[0] = __builtin_bit_cast(bf16x8, x.h);
    t[1] = __builtin_bit_cast(bf16x8, x.m);
    t[2] = __builtin_bit_cast(bf16x8, x.l);
}
__device__ __forceinline__ void to_terms(const __bf16* p, bf16x8 (&t)[1]) { t[0] = *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ void to_terms(const float* p, bf16x8 (&t)[3]) { as_terms(split8(*reinterpret_cast<const Four*>(p), *reinterpret_cast<const Four*>(p + 4)), t); }
__device__ __forceinline__ void to_terms(const float (&w)[8], bf16x8 (&t)[1])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) t[0][i] = (__bf16)w[i];
}
__device__ __forceinline__ void to_terms(const float (&w)[8], bf16x8 (&t)[3])
{
    Terms x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.set_pair(i, w[2 * i], w[2 * i + 1]);
    as_terms(x, t);
}
// Eight weights added to the normaliser as the value product takes them, rounded where they are one term: an error that they share is then in both
// sums, and cancels.
template <int kWeightTerms>
__device__ __forceinline__ float add_weights(float sum, const float (&p)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        if constexpr (kWeightTerms == 1)
            sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{(__bf16)p[i], (__bf16)p[i + 1]}, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, sum, false);
        else
            sum += p[i] + p[i + 1];
    }
    return sum;
}
template <int kTerms>
__device__ __forceinline__ void no_terms(bf16x8 (&t)[kTerms])
{
#pragma unroll
    for (int i = 0; i < kTerms; ++i) t[i] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

// Where a 16-token group of KV head g stands in the pools, in units of 256 bytes, and in the exponents, in units of 16: 32 bits for pools of
// a terabyte.  (Byte offsets are 64-bit products, which took the loops of the attention kernels up to 60 scalar instructions a step.)
struct Where { uint32_t data, exps; };
struct Finder {
    uint32_t page_data, page_exps, data0, exps0, group;
    __device__ __forceinline__ Finder(const CacheView& c, int d, int g)
        : page_data((uint32_t)c.hkv * (uint32_t)(d * c.ps >> 8)), page_exps((uint32_t)c.hkv * (uint32_t)(c.ps >> 3)),
          data0((uint32_t)g * (uint32_t)(d * c.ps >> 8)), exps0((uint32_t)g * (uint32_t)(c.ps >> 3)), group((uint32_t)d >> 4) {}
    // group gi of the page
    __device__ __forceinline__ Where at(int page, int gi) const
    {
        return Where{(uint32_t)page * page_data + data0 + (uint32_t)gi * group, (uint32_t)page * page_exps + exps0 + (uint32_t)gi};
    }
};
__device__ __forceinline__ const uint8_t* data_at(const void* pool, uint32_t data) { return (const uint8_t*)pool + ((uint64_t)data << 8); }
__device__ __forceinline__ const uint8_t* exps_at(const uint8_t* exps, uint32_t at) { return exps + ((uint64_t)at << 4); }

// A weight of zero does not hide a NaN.  Where some of a workgroup's columns do not see a tile whole, prefill takes NaN among its values as
// zeros and afterwards, if there was one, this takes them to the columns that do see them, byte by byte: tokens first .. last of session s,
// o[mb][i] being channel mb * 32 + (i / 4) * 8 + hi * 4 + i % 4 of the lane's column, which sees positions up to qpos.
template <int kMb, class O>
__device__ __forceinline__ void nan_to_those_that_see_it(const AttnArgs& a, const Finder& find, int s, int first, int last, int qpos, int hi, O (&o)[kMb])
{
#pragma unroll 1
    for (int at = first; at <= last; ++at) {
        const Where w = find.at(a.bt[(int64_t)s * a.max_pages + (at >> a.c.ps_shift)], (at & (a.c.ps - 1)) >> 4);
        const uint8_t* vp = data_at(a.c.v, w.data) + (at & 15) + hi * 64;
#pragma unroll
        for (int mb = 0; mb < kMb; ++mb)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (mb * 32 + q * 8 >= a.c.d) break;             // (a branch also where the caller knows better: fewer loads in flight, fewer registers)
#pragma unroll
                for (int i = q * 4; i < q * 4 + 4; ++i)
                    o[mb][i] = at <= qpos && (vp[(mb * 32 + q * 8 + (i & 3)) * 16] & 0x7F) == 0x7F ? __builtin_nanf("") : o[mb][i];
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// K and V are read once by a decode step: the streaming hint
__device__ __forceinline__ u32x4 stream16(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }

}  // namespace q8
}  // namespace ag
