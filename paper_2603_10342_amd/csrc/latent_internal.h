// Internal declarations of the latent cache (include/ag_latent.h): its geometry, the launchers, and how a batch's work is dealt.
#pragma once

#include "ag_latent.h"
#include "rope_internal.h"

namespace ag {
namespace latent {

constexpr int row_of(int latent_dim, int rope_dim) { return (latent_dim + rope_dim + 63) / 64 * 64; }

struct Cache {                  // host-validated view
    void* pool;
    int num_pages, ps, ps_shift, lat, rd;
};

struct AppendArgs {
    Cache c;
    rope::Spec r;               // r.turns == nullptr: rows that are rotated already
    bool pairs;
    const void* lat;
    int64_t lat_stride;
    const void* rot;
    int64_t rot_stride;
    const int32_t* bt;
    int max_pages;
    const int32_t *prefix_lens, *new_lens, *cu_new;
    int batch, total;
};
ag_status launch_append(const AppendArgs& a, hipStream_t st);

// An attention problem.  Decode: ctx_lens, one row a session.  Otherwise rows through cu_new.
struct AttnArgs {
    Cache c;
    const void* q;
    void* out;
    const int32_t* bt;
    int max_pages;
    const int32_t *prefix_lens, *new_lens, *cu_new, *ctx_lens;
    int batch, total, max_new, max_ctx, heads;
    float scale;
    void* ws;
};
// Bytes of workspace; 0 for a problem that one launch cannot hold.
size_t    attn_workspace(bool decode, int batch, int total, int heads, int lat, int max_ctx);
ag_status launch_attn(const AttnArgs& a, hipStream_t st);

}  // namespace latent
}  // namespace ag
