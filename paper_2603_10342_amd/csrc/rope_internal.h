// Rotary positions: what the kernels that rotate rows share (include/ag_rope.h).  Internal.
#pragma once

#include "ag_internal.h"
#include "ag_rope.h"

namespace ag {
namespace rope {

// Checks an ag_rope; `most` is the widest rotated part the call can take.
ag_status check(const ag_rope* rope, int most);

struct Spec {                   // an ag_rope as the kernels see it
    const double* turns;
    int half;                   // rot_dim / 2 pairs
    float magnitude;
    bool transposed;            // the sine with the other sign
};
inline Spec spec_of(const ag_rope& r, bool transposed = false) { return Spec{r.turns, r.rot_dim / 2, r.magnitude, transposed}; }

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// m cos and m sin of 2 pi pos turns, in 64 bits up to their last rounding: 32 lose a far position's angle (2^20 positions of a radian each are off by 2^-4).  The whole
// turns go first, then the nearest quarter; what is left, |x| <= pi / 4, is inside the series' first terms (the first left out: x^13 / 13! < 2^-36 of the sine,
// x^12 / 12! < 2^-33).  About twenty 64-bit operations a pair and token, shared by all heads.
__device__ __forceinline__ f32x2 cos_sin(int pos, const Spec& r, int i)
{
    const double t = r.turns[i], a = fma((double)pos, t, -rint((double)pos * t));         // (the product unrounded)
    const double quarter = rint(4.0 * a), x = (a - 0.25 * quarter) * 6.283185307179586477, xx = x * x;
    const double s = x * fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
    const double c = fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, -1.0 / 3628800, 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
    const int k = (int)quarter & 3;
    const double m = r.magnitude, cosine = (k & 1) ? s : c, sine = (k & 1) ? c : s;
    return f32x2{(float)((k == 1 || k == 2) ? -m * cosine : m * cosine), (float)(((k >= 2) != r.transposed) ? -m * sine : m * sine)};
}

__device__ __forceinline__ void turn(float& a, float& b, f32x2 cs)
{
    const float x = fmaf(a, cs[0], -(b * cs[1])), y = fmaf(b, cs[0], a * cs[1]);       // (written out: every kernel gives the same bits)
    a = x;
    b = y;
}

// Eight channels of a row: 16 bytes of bf16, 32 of fp32.
template <typename A>
struct alignas(16) Eight { u32x4 w[sizeof(A) / 2]; };

__device__ __forceinline__ void widen(const Eight<__bf16>& r, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __builtin_bit_cast(float, r.w[0][i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, r.w[0][i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void widen(const Eight<float>& r, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)r.w[i >> 2][i & 3]);
}
__device__ __forceinline__ uint32_t pair_of(float a, float b)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, pair{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ void narrow(const float (&x)[8], Eight<__bf16>& r)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[0][i] = pair_of(x[2 * i], x[2 * i + 1]);
}
__device__ __forceinline__ void narrow(const float (&x)[8], Eight<float>& r)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = __builtin_bit_cast(uint32_t, x[i]);
}

// A lane's share of a row: sixteen channels in two runs of eight that hold eight whole pairs, or sixteen (or the last eight) of those that stay.
template <typename A>
struct Unit { Eight<A> lo, hi; };

struct Units {                  // how a row of d channels is cut
    int d, half, rotated;       // the first `rotated` units turn
    __host__ __device__ Units(int d_, int half_) : d(d_), half(half_), rotated(half_ >> 3) {}
    __host__ __device__ int count() const { return rotated + (d - 2 * half + 15) / 16; }
    template <bool kPairs>
    __device__ __forceinline__ int lo(int u) const { return kPairs || u >= rotated ? u * 16 - (u >= rotated ? rotated * 16 - 2 * half : 0) : u * 8; }
    template <bool kPairs>
    __device__ __forceinline__ int hi(int u) const { return kPairs || u >= rotated ? lo<kPairs>(u) + 8 : half + u * 8; }
};

template <bool kPairs, typename A>
__device__ __forceinline__ void load_unit(const Units& us, const A* row, int u, Unit<A>& r)
{
    const int lo = us.lo<kPairs>(u), hi = us.hi<kPairs>(u);
    r.lo = *reinterpret_cast<const Eight<A>*>(row + lo);
    if (hi < us.d) r.hi = *reinterpret_cast<const Eight<A>*>(row + hi);
}
// cs: the cosines and sines of the row's position
template <bool kPairs, typename A>
__device__ __forceinline__ void turn_unit(const Units& us, int u, const f32x2* cs, Unit<A>& r)
{
    if (u >= us.rotated) return;
    float a[8], b[8];
    widen(r.lo, a);
    widen(r.hi, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (!kPairs) turn(a[i], b[i], cs[u * 8 + i]);
        else if (i < 4) turn(a[2 * i], a[2 * i + 1], cs[u * 8 + i]);
        else turn(b[2 * i - 8], b[2 * i - 7], cs[u * 8 + i]);
    }
    narrow(a, r.lo);
    narrow(b, r.hi);
}
// kStream: with the streaming hint
template <bool kStream = false, typename A>
__device__ __forceinline__ void store_eight(A* dst, const Eight<A>& r)
{
    if constexpr (kStream) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(A) / 2; ++i) __builtin_nontemporal_store(r.w[i], reinterpret_cast<u32x4*>(dst) + i);
    } else {
        *reinterpret_cast<Eight<A>*>(dst) = r;
    }
}
template <bool kPairs, bool kStream = false, typename A>
__device__ __forceinline__ void store_unit(const Units& us, A* row, int u, const Unit<A>& r)
{
    const int lo = us.lo<kPairs>(u), hi = us.hi<kPairs>(u);
    store_eight<kStream>(row + lo, r.lo);
    if (hi < us.d) store_eight<kStream>(row + hi, r.hi);
}

struct RowsArgs {
    Spec r;
    int layout, dtype;
    const void* x;
    int64_t xt, xh;
    void* y;
    int64_t yt, yh;
    int heads, d;
    const int32_t *prefix_lens, *new_lens, *cu_new;
    int batch, total;
};
ag_status launch_rows(const RowsArgs& a, hipStream_t st);

struct AppendArgs {
    CacheView c;
    Spec r;
    int layout;
    const void* q;              // nullptr: no queries
    void* q_out;
    int hq;
    const void *k_new, *v_new;
    const int32_t* bt;
    int max_pages;
    const int32_t *prefix_lens, *new_lens, *cu_new;
    int batch, total;
};
ag_status launch_append(const AppendArgs& a, hipStream_t st);

}  // namespace rope
}  // namespace ag
