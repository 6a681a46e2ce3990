// Append to the latent cache (include/ag_latent.h): latent channels copied, rotary ones rotated on the way, a contiguous row of the pool a token.
//
// Bound by HBM, 2 T (L + R) 2 bytes, or for a decode step's few rows (4.1 us) by three dependent memory round trips: lengths, page, store.  A wave takes one token
// of 512 channels, two of fewer, and deals its lanes to all their 16-byte pieces, then to all their rotary pairs; rows are requested before their sessions are
// looked up.  32768 rows of 512 + 64 channels 14.3 us, 5.3 TB/s, with four tokens a wave the same; 107000 of 256 + 32 23 us, with one 29; 195000 of 128 + 64 41 us,
// with one 59, with four 48 (and a step of 1024 sessions 4.1 us, with four 10.6: each looks for its session).
#include "find_session.h"
#include "latent_internal.h"

namespace ag {
namespace latent {
namespace {

using rope::f32x2;
using rope::u32x4;

// kPieces: 16-byte pieces of a row's latent part; kPairs: its rotary pairs
template <int kPieces, int kPairs>
__global__ __launch_bounds__(256) void append_latent_kernel(AppendArgs x)
{
    constexpr int kTok = kPieces == 64 ? 1 : 2, kTurns = (kTok * kPairs + 63) / 64, kRow = row_of(kPieces * 8, kPairs * 2);
    const int lane = threadIdx.x & 63, t0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kTok;
    if (t0 >= x.total) return;
    const int most = min(kTok, x.total - t0);                          // tokens of this wave
    u32x4 lat = {};
    __bf16 a[kTurns], b[kTurns];
    auto first = [&](int pair) { return x.pairs ? 2 * pair : pair; };
    auto second = [&](int pair) { return x.pairs ? 2 * pair + 1 : pair + kPairs; };
    const int mine = lane / kPieces, piece = lane % kPieces;
    if (mine < most) lat = *reinterpret_cast<const u32x4*>((const __bf16*)x.lat + (int64_t)(t0 + mine) * x.lat_stride + piece * 8);
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int at = i * 64 + lane, tok = at / kPairs, pair = at % kPairs;
        if (tok < most) {
            const __bf16* const row = (const __bf16*)x.rot + (int64_t)(t0 + tok) * x.rot_stride;
            a[i] = row[first(pair)];
            b[i] = row[second(pair)];
        }
    }
    int pos[kTok];                                                     // uniform, like the rows
    int64_t row[kTok];
    Session f = {0, 0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
        const int t = t0 + j;
        pos[j] = -1;
        row[j] = 0;
        if (j < most) {
            if (j == 0 || t >= f.row0 + f.new_len) f = find_session(x.new_lens, x.prefix_lens, x.cu_new, x.batch, t, [](int, int cu) { return cu; });
            if (t - f.row0 < f.new_len) {                              // (otherwise behind the last session: nobody's)
                pos[j] = f.prefix + (t - f.row0);
                row[j] = (int64_t)x.bt[(int64_t)f.s * x.max_pages + (pos[j] >> x.c.ps_shift)] * x.c.ps + (pos[j] & (x.c.ps - 1));
            }
        }
    }
    auto pick = [&](const auto& of, int tok) {
        auto r = of[0];
#pragma unroll
        for (int j = 1; j < kTok; ++j) r = tok == j ? of[j] : r;
        return r;
    };
    __bf16* const pool = (__bf16*)x.c.pool;
    if (mine < most && pick(pos, mine) >= 0) *reinterpret_cast<u32x4*>(pool + pick(row, mine) * kRow + piece * 8) = lat;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int at = i * 64 + lane, tok = at / kPairs, pair = at % kPairs, p = pick(pos, tok);
        if (tok >= most || p < 0) continue;
        if (x.r.turns) {
            float u = (float)a[i], v = (float)b[i];
            rope::turn(u, v, rope::cos_sin(p, x.r, pair));
            a[i] = (__bf16)u;
            b[i] = (__bf16)v;
        }
        __bf16* const dst = pool + pick(row, tok) * kRow + kPieces * 8;
        dst[first(pair)] = a[i];
        dst[second(pair)] = b[i];
    }
}

template <int kPieces, int kPairs>
ag_status run(const AppendArgs& a, hipStream_t st)
{
    constexpr int kTok = kPieces == 64 ? 4 : 8;                        // of a workgroup
    hipLaunchKernelGGL((append_latent_kernel<kPieces, kPairs>), dim3((a.total + kTok - 1) / kTok), dim3(256), 0, st, a);
    return hip_check(hipGetLastError(), "append launch");
}
template <int kPieces>
ag_status run(const AppendArgs& a, hipStream_t st) { return a.c.rd == 64 ? run<kPieces, 32>(a, st) : run<kPieces, 16>(a, st); }

}  // namespace

ag_status launch_append(const AppendArgs& a, hipStream_t st)
{
    return a.c.lat == 512 ? run<64>(a, st) : a.c.lat == 256 ? run<32>(a, st) : run<16>(a, st);
}

}  // namespace latent
}  // namespace ag
