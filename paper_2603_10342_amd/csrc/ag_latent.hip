// C-ABI entry points of the latent cache: argument validation, as ag_api.hip does it for the others (see include/ag_latent.h).
#include "latent_internal.h"

namespace ag {
namespace latent {
namespace {

bool aligned(const void* p) { return (uintptr_t)p % 16 == 0; }
bool width_known(int lat, int rd) { return (lat == 128 || lat == 256 || lat == 512) && (rd == 32 || rd == 64); }

ag_status view(const ag_latent_cache* c, Cache* v)
{
    if (!c) { set_error("cache is NULL"); return AG_ERR_INVALID_ARG; }
    if (!c->pool) { set_error("cache pool is NULL"); return AG_ERR_INVALID_ARG; }
    if (c->num_pages <= 0) { set_error("num_pages=%d must be positive", c->num_pages); return AG_ERR_INVALID_ARG; }
    if (!width_known(c->latent_dim, c->rope_dim)) {
        set_error("latent_dim %d with rope_dim %d unsupported (128, 256 or 512 with 32 or 64)", c->latent_dim, c->rope_dim);
        return AG_ERR_UNSUPPORTED;
    }
    int shift = 4;
    while (shift < 8 && (1 << shift) != c->page_size) ++shift;
    if ((1 << shift) != c->page_size) {
        set_error("page_size %d unsupported by a latent cache (power of two from 16 to 256)", c->page_size);
        return AG_ERR_UNSUPPORTED;
    }
    if (!aligned(c->pool)) { set_error("the pool must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    *v = Cache{c->pool, c->num_pages, c->page_size, shift, c->latent_dim, c->rope_dim};
    return AG_OK;
}

// Positions are 32-bit numbers, and those of the steps after the last one too.
constexpr int kMostCtx = 0x7fffffff - 1024;

ag_status attend(bool decode, const ag_latent_cache* cache, const void* q, void* out, const int32_t* bt, int max_pages, const int32_t* prefix_lens,
                 const int32_t* new_lens, const int32_t* cu_new, const int32_t* ctx_lens, int batch, int total, int max_new, int max_ctx, int heads,
                 float scale, void* ws, size_t ws_bytes, void* stream)
{
    AttnArgs a;
    ag_status st = view(cache, &a.c);
    if (st) return st;
    if (!q || !out || !bt || (decode ? !ctx_lens : !prefix_lens || !new_lens || !cu_new)) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || max_pages <= 0 || total < 0 || max_new < 0 || max_ctx < 0) {
        set_error("batch=%d max_pages_per_seq=%d total_new=%d max_new=%d max_ctx=%d: sizes must be positive", batch, max_pages, total, max_new, max_ctx);
        return AG_ERR_INVALID_ARG;
    }
    if (!aligned(q) || !aligned(out)) { set_error("q and out must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    if (heads <= 0) { set_error("num_q_heads %d must be positive", heads); return AG_ERR_INVALID_ARG; }
    if (!(scale > 0.0f) || !(scale < 1e30f)) { set_error("scale must be positive and finite"); return AG_ERR_INVALID_ARG; }
    if (max_ctx > kMostCtx) { set_error("max_ctx %d exceeds %d", max_ctx, kMostCtx); return AG_ERR_INVALID_ARG; }
    if ((int64_t)max_ctx > (int64_t)max_pages * a.c.ps) {
        set_error("max_ctx %d exceeds max_pages_per_seq * page_size = %lld", max_ctx, (long long)max_pages * a.c.ps);
        return AG_ERR_INVALID_ARG;
    }
    if (max_new > total) { set_error("max_new %d exceeds total_new %d", max_new, total); return AG_ERR_INVALID_ARG; }
    if (!decode && max_ctx < max_new) { set_error("max_ctx %d is smaller than max_new %d", max_ctx, max_new); return AG_ERR_INVALID_ARG; }
    if (total == 0 || max_new == 0) return AG_OK;
    const size_t need = attn_workspace(decode, batch, total, heads, a.c.lat, max_ctx);
    if (!need) { set_error("the batch is too large for one launch (rows times heads times context)"); return AG_ERR_INVALID_ARG; }
    if (ws_bytes < need || !ws) { set_error("workspace too small: %zu bytes given, %zu needed", ws_bytes, need); return AG_ERR_WORKSPACE; }
    if (!aligned(ws)) { set_error("the workspace must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    a.q = q; a.out = out; a.bt = bt; a.max_pages = max_pages;
    a.prefix_lens = prefix_lens; a.new_lens = new_lens; a.cu_new = cu_new; a.ctx_lens = ctx_lens;
    a.batch = batch; a.total = total; a.max_new = max_new; a.max_ctx = max_ctx; a.heads = heads; a.scale = scale; a.ws = ws;
    return launch_attn(a, (hipStream_t)stream);
}

}  // namespace
}  // namespace latent
}  // namespace ag

using namespace ag;

extern "C" {

int32_t ag_latent_row(int32_t latent_dim, int32_t rope_dim) { return latent::width_known(latent_dim, rope_dim) ? latent::row_of(latent_dim, rope_dim) : 0; }

ag_status ag_kv_append_latent(const ag_latent_cache* cache, const ag_rope* rope, const void* latent_new, int64_t latent_stride, const void* rope_new,
                              int64_t rope_stride, const int32_t* block_tables, int32_t max_pages_per_seq, const int32_t* prefix_lens,
                              const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new, void* stream)
{
    latent::AppendArgs a;
    ag_status st = latent::view(cache, &a.c);
    if (st) return st;
    if (rope) {
        if ((st = rope::check(rope, a.c.rd))) return st;
        if (rope->rot_dim != a.c.rd) { set_error("rot_dim %d is not the cache's rope_dim %d", rope->rot_dim, a.c.rd); return AG_ERR_INVALID_ARG; }
    }
    if (!latent_new || !rope_new || !block_tables || !prefix_lens || !new_lens || !cu_new) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || max_pages_per_seq <= 0 || total_new < 0) {
        set_error("batch=%d max_pages_per_seq=%d total_new=%d: sizes must be positive", batch, max_pages_per_seq, total_new);
        return AG_ERR_INVALID_ARG;
    }
    const int64_t most = INT64_MAX >> 34;                             // (the last row's offset in bytes fits 64 bits)
    for (int64_t s : {latent_stride, rope_stride})
        if (s < 0 || s > most || s % 8) { set_error("strides must be multiples of 8 elements and not negative"); return AG_ERR_INVALID_ARG; }
    if (!latent::aligned(latent_new) || !latent::aligned(rope_new)) { set_error("latent_new and rope_new must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    if (total_new == 0) return AG_OK;
    if ((total_new + 3ll) / 4 > 0xFFFFFFFFll / 256) { set_error("total_new=%d: too many rows for one launch", total_new); return AG_ERR_INVALID_ARG; }
    a.r = rope ? rope::spec_of(*rope) : rope::Spec{nullptr, a.c.rd / 2, 1.0f, false};
    a.pairs = rope && rope->layout == AG_ROPE_PAIRS;
    a.lat = latent_new; a.lat_stride = latent_stride; a.rot = rope_new; a.rot_stride = rope_stride;
    a.bt = block_tables; a.max_pages = max_pages_per_seq; a.prefix_lens = prefix_lens; a.new_lens = new_lens; a.cu_new = cu_new;
    a.batch = batch; a.total = total_new;
    return latent::launch_append(a, (hipStream_t)stream);
}

size_t ag_attn_decode_latent_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t latent_dim, int32_t max_ctx)
{
    if (batch <= 0 || num_q_heads <= 0 || !latent::width_known(latent_dim, 64) || max_ctx < 0 || max_ctx > latent::kMostCtx) return 0;
    return latent::attn_workspace(true, batch, batch, num_q_heads, latent_dim, max_ctx);
}

ag_status ag_attn_decode_latent(const ag_latent_cache* cache, const void* q, void* out, const int32_t* block_tables, int32_t max_pages_per_seq,
                                const int32_t* ctx_lens, int32_t batch, int32_t max_ctx, int32_t num_q_heads, float scale, void* workspace,
                                size_t workspace_bytes, void* stream)
{
    return latent::attend(true, cache, q, out, block_tables, max_pages_per_seq, nullptr, nullptr, nullptr, ctx_lens, batch, batch, batch > 0 ? 1 : 0, max_ctx,
                          num_q_heads, scale, workspace, workspace_bytes, stream);
}

size_t ag_attn_resume_latent_workspace_bytes(int32_t batch, int32_t total_new, int32_t num_q_heads, int32_t latent_dim, int32_t max_ctx)
{
    if (batch <= 0 || total_new < 0 || num_q_heads <= 0 || !latent::width_known(latent_dim, 64) || max_ctx < 0 || max_ctx > latent::kMostCtx) return 0;
    return latent::attn_workspace(false, batch, total_new, num_q_heads, latent_dim, max_ctx);
}

ag_status ag_attn_resume_latent(const ag_latent_cache* cache, const void* q, void* out, const int32_t* block_tables, int32_t max_pages_per_seq,
                                const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new,
                                int32_t max_new, int32_t max_ctx, int32_t num_q_heads, float scale, void* workspace, size_t workspace_bytes, void* stream)
{
    return latent::attend(false, cache, q, out, block_tables, max_pages_per_seq, prefix_lens, new_lens, cu_new, nullptr, batch, total_new, max_new, max_ctx,
                          num_q_heads, scale, workspace, workspace_bytes, stream);
}

}  // extern "C"
