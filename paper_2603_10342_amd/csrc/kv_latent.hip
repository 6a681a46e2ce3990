// Append to the latent cache (include/ag_latent.h): latent channels copied, rotary ones rotated on the way, a contiguous row of the pool a token.
//
// Bound by HBM, 2 T (L + R) 2 bytes, or for a decode step's few rows by three dependent memory round trips: lengths, page, store.  A wave takes kTok consecutive
// tokens: their rows are requested before their sessions are looked up.  A lane holds 16 bytes of the latent part and one rotary pair.
#include "find_session.h"
#include "latent_internal.h"

namespace ag {
namespace latent {
namespace {

using rope::f32x2;
using rope::u32x4;

template <int kTok>
__global__ __launch_bounds__(256) void append_latent_kernel(AppendArgs x)
{
    const int lane = threadIdx.x & 63, t0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kTok;
    if (t0 >= x.total) return;
    const int row = row_of(x.c.lat, x.c.rd), half = x.c.rd / 2;
    const int ca = x.pairs ? 2 * lane : lane, cb = x.pairs ? 2 * lane + 1 : lane + half;          // the lane's pair
    u32x4 lat[kTok];
    __bf16 a[kTok], b[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        const int64_t t = min(t0 + j, x.total - 1);
        if (lane * 8 < x.c.lat) lat[j] = *reinterpret_cast<const u32x4*>((const __bf16*)x.lat + t * x.lat_stride + lane * 8);
        if (lane < half) {
            a[j] = ((const __bf16*)x.rot)[t * x.rot_stride + ca];
            b[j] = ((const __bf16*)x.rot)[t * x.rot_stride + cb];
        }
    }
    Session f = {0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        const int t = t0 + j;
        if (t >= x.total) break;
        if (j == 0 || t >= f.row0 + f.new_len) f = find_session(x.new_lens, x.prefix_lens, x.cu_new, x.batch, t, [](int, int cu) { return cu; });
        if (t - f.row0 >= f.new_len) break;                            // behind the last session: nobody's, like all that follow
        const int pos = f.prefix + (t - f.row0);
        const int64_t page = x.bt[(int64_t)f.s * x.max_pages + (pos >> x.c.ps_shift)];
        __bf16* const dst = (__bf16*)x.c.pool + (page * x.c.ps + (pos & (x.c.ps - 1))) * row;
        if (lane * 8 < x.c.lat) *reinterpret_cast<u32x4*>(dst + lane * 8) = lat[j];
        if (lane < half) {
            __bf16 ra = a[j], rb = b[j];
            if (x.r.turns) {
                float u = (float)ra, v = (float)rb;
                rope::turn(u, v, rope::cos_sin(pos, x.r, lane));
                ra = (__bf16)u;
                rb = (__bf16)v;
            }
            dst[x.c.lat + ca] = ra;
            dst[x.c.lat + cb] = rb;
        }
    }
}

}  // namespace

ag_status launch_append(const AppendArgs& a, hipStream_t st)
{
    // One token a wave while the chip holds them all at once
    if (a.total <= 4096) hipLaunchKernelGGL(append_latent_kernel<1>, dim3((a.total + 3) / 4), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(append_latent_kernel<4>, dim3((a.total + 15) / 16), dim3(256), 0, st, a);
    return hip_check(hipGetLastError(), "append launch");
}

}  // namespace latent
}  // namespace ag
