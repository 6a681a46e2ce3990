// C-ABI entry points of the 8-bit cache: argument validation, as ag_api.hip does it for the others (see include/ag_q8.h).
#include "q8_internal.h"

namespace ag {
namespace q8 {
namespace {

bool aligned(const void* p) { return (uintptr_t)p % 16 == 0; }

ag_status view(const ag_kv_cache_q8* c, CacheView* v)
{
    if (!c) { set_error("cache is NULL"); return AG_ERR_INVALID_ARG; }
    if (!c->k_pool || !c->v_pool || !c->exps) { set_error("cache pools or exponents are NULL"); return AG_ERR_INVALID_ARG; }
    if (c->num_pages <= 0 || c->num_kv_heads <= 0) {
        set_error("num_pages=%d num_kv_heads=%d must be positive", c->num_pages, c->num_kv_heads);
        return AG_ERR_INVALID_ARG;
    }
    if (c->dtype != AG_F32 && c->dtype != AG_BF16) { set_error("dtype %d unsupported", c->dtype); return AG_ERR_UNSUPPORTED; }
    if (c->head_dim <= 0 || c->head_dim > 256 || c->head_dim % 16) {
        set_error("head_dim %d unsupported by an 8-bit cache (multiple of 16, at most 256)", c->head_dim);
        return AG_ERR_UNSUPPORTED;
    }
    int shift = 4;
    while (shift < 8 && (1 << shift) != c->page_size) ++shift;
    if ((1 << shift) != c->page_size) {
        set_error("page_size %d unsupported by an 8-bit cache (power of two from 16 to 256)", c->page_size);
        return AG_ERR_UNSUPPORTED;
    }
    if (!aligned(c->k_pool) || !aligned(c->v_pool) || !aligned(c->exps)) {
        set_error("the pools and exps must be 16-byte aligned");
        return AG_ERR_INVALID_ARG;
    }
    v->k = c->k_pool; v->v = c->v_pool;
    v->num_pages = c->num_pages; v->ps = c->page_size; v->ps_shift = shift;
    v->hkv = c->num_kv_heads; v->d = c->head_dim; v->dtype = c->dtype;
    return AG_OK;
}

// Positions are 32-bit numbers, and those of the steps after the last one too.
constexpr int kMostCtx = 0x7fffffff - 1024;

// q and out of every attention call, the heads, the scale and the longest context
ag_status check_attention(const CacheView& c, const void* q, const void* out, int hq, float scale, int max_ctx, int max_pages)
{
    if (!aligned(q) || !aligned(out)) { set_error("q and out must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    if (hq <= 0 || hq % c.hkv) {
        set_error("num_q_heads %d is not a positive multiple of num_kv_heads %d", hq, c.hkv);
        return AG_ERR_INVALID_ARG;
    }
    if (!(scale > 0.0f) || !(scale < 1e30f)) { set_error("scale must be positive and finite"); return AG_ERR_INVALID_ARG; }
    if (max_ctx > kMostCtx) { set_error("max_ctx %d exceeds %d", max_ctx, kMostCtx); return AG_ERR_INVALID_ARG; }
    if ((int64_t)max_ctx > (int64_t)max_pages * c.ps) {
        set_error("max_ctx %d exceeds max_pages_per_seq * page_size = %lld", max_ctx, (long long)max_pages * c.ps);
        return AG_ERR_INVALID_ARG;
    }
    return AG_OK;
}

// Append and read-back take the same arguments; the rows are the caller's input or its output.
ag_status rows_common(const ag_kv_cache_q8* cache, const void* k, const void* v, const int32_t* bt, int max_pages, const int32_t* prefix_lens,
                      const int32_t* new_lens, const int32_t* cu_new, int batch, int total, CacheView* c)
{
    ag_status st = view(cache, c);
    if (st) return st;
    if (!k || !v || !bt || !prefix_lens || !new_lens || !cu_new) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || max_pages <= 0 || total < 0) {
        set_error("batch=%d max_pages_per_seq=%d total_new=%d: sizes must be positive", batch, max_pages, total);
        return AG_ERR_INVALID_ARG;
    }
    if (!aligned(k) || !aligned(v)) { set_error("rows of keys and values must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    return AG_OK;
}

ag_status prefill_common(const ag_kv_cache_q8* cache, const void* q, void* out, const int32_t* bt, int max_pages, const int32_t* prefix_lens,
                         bool need_prefix, const int32_t* new_lens, const int32_t* cu_new, int batch, int total_new, int max_new, int max_ctx,
                         int hq, float scale, void* stream)
{
    Args x;
    AttnArgs& a = x.a;
    ag_status st = view(cache, &a.c);
    if (st) return st;
    if (!q || !out || !bt || !new_lens || !cu_new || (need_prefix && !prefix_lens)) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || max_pages <= 0 || total_new < 0 || max_new < 0) {
        set_error("batch=%d max_pages_per_seq=%d total_new=%d max_new=%d: sizes must be positive", batch, max_pages, total_new, max_new);
        return AG_ERR_INVALID_ARG;
    }
    if ((st = check_attention(a.c, q, out, hq, scale, max_ctx, max_pages))) return st;
    if (max_new > total_new) { set_error("max_new %d exceeds total_new %d", max_new, total_new); return AG_ERR_INVALID_ARG; }
    if (max_ctx < max_new) { set_error("max_ctx %d is smaller than max_new %d", max_ctx, max_new); return AG_ERR_INVALID_ARG; }
    if (total_new == 0 || max_new == 0) return AG_OK;
    x.exps = (const uint8_t*)cache->exps;
    a.q = q; a.out = out; a.bt = bt; a.max_pages = max_pages;
    a.prefix_lens = prefix_lens; a.new_lens = new_lens; a.cu_new = cu_new; a.ctx_lens = nullptr;
    a.batch = batch; a.total_rows = total_new; a.max_new = max_new; a.max_ctx = max_ctx; a.hq = hq; a.scale = scale;
    return launch_prefill(x, (hipStream_t)stream);
}

}  // namespace
}  // namespace q8
}  // namespace ag

using namespace ag;

extern "C" {

ag_status ag_kv_append_q8(const ag_kv_cache_q8* cache, const void* k_new, const void* v_new, const int32_t* block_tables,
                          int32_t max_pages_per_seq, const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                          int32_t batch, int32_t total_new, void* stream)
{
    CacheView c;
    ag_status st = q8::rows_common(cache, k_new, v_new, block_tables, max_pages_per_seq, prefix_lens, new_lens, cu_new, batch, total_new, &c);
    if (st || total_new == 0) return st;
    return q8::launch_append(c, (uint8_t*)cache->exps, k_new, v_new, block_tables, max_pages_per_seq, prefix_lens, new_lens, cu_new, batch,
                             total_new, (hipStream_t)stream);
}

ag_status ag_kv_read_q8(const ag_kv_cache_q8* cache, void* k_out, void* v_out, const int32_t* block_tables, int32_t max_pages_per_seq,
                        const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new,
                        void* stream)
{
    CacheView c;
    ag_status st = q8::rows_common(cache, k_out, v_out, block_tables, max_pages_per_seq, prefix_lens, new_lens, cu_new, batch, total_new, &c);
    if (st || total_new == 0) return st;
    return q8::launch_read(c, (const uint8_t*)cache->exps, k_out, v_out, block_tables, max_pages_per_seq, prefix_lens, new_lens, cu_new, batch,
                           total_new, (hipStream_t)stream);
}

ag_status ag_attn_prefill_q8(const ag_kv_cache_q8* cache, const void* q, void* out, const int32_t* block_tables, int32_t max_pages_per_seq,
                             const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new, int32_t max_new,
                             int32_t num_q_heads, float scale, void* stream)
{
    return q8::prefill_common(cache, q, out, block_tables, max_pages_per_seq, nullptr, false, new_lens, cu_new, batch, total_new, max_new,
                              max_new, num_q_heads, scale, stream);
}

ag_status ag_attn_resume_q8(const ag_kv_cache_q8* cache, const void* q, void* out, const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new,
                            int32_t max_new, int32_t max_ctx, int32_t num_q_heads, float scale, void* stream)
{
    return q8::prefill_common(cache, q, out, block_tables, max_pages_per_seq, prefix_lens, true, new_lens, cu_new, batch, total_new, max_new,
                              max_ctx, num_q_heads, scale, stream);
}

size_t ag_attn_decode_q8_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t head_dim, int32_t max_ctx)
{
    if (batch <= 0 || num_q_heads <= 0 || head_dim <= 0 || max_ctx < 0 || max_ctx > q8::kMostCtx) return 0;
    return q8::decode_workspace(batch, num_q_heads, head_dim, max_ctx);
}

ag_status ag_attn_decode_q8(const ag_kv_cache_q8* cache, const void* q, void* out, const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* ctx_lens, int32_t batch, int32_t max_ctx, int32_t num_q_heads, float scale, void* workspace,
                            size_t workspace_bytes, void* stream)
{
    q8::Args x;
    AttnArgs& a = x.a;
    ag_status st = q8::view(cache, &a.c);
    if (st) return st;
    if (!q || !out || !block_tables || !ctx_lens) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || max_pages_per_seq <= 0 || max_ctx < 0) {
        set_error("batch=%d max_pages_per_seq=%d max_ctx=%d: sizes must be positive", batch, max_pages_per_seq, max_ctx);
        return AG_ERR_INVALID_ARG;
    }
    if ((st = q8::check_attention(a.c, q, out, num_q_heads, scale, max_ctx, max_pages_per_seq))) return st;
    const size_t need = q8::decode_workspace(batch, num_q_heads, a.c.d, max_ctx);
    if (workspace_bytes < need || !workspace) {
        set_error("decode workspace too small: %zu bytes given, %zu needed", workspace_bytes, need);
        return AG_ERR_WORKSPACE;
    }
    if (!q8::aligned(workspace)) { set_error("decode workspace must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    x.exps = (const uint8_t*)cache->exps;
    a.q = q; a.out = out; a.bt = block_tables; a.max_pages = max_pages_per_seq;
    a.prefix_lens = nullptr; a.new_lens = nullptr; a.cu_new = nullptr; a.ctx_lens = ctx_lens;
    a.batch = batch; a.total_rows = batch; a.max_new = 1; a.max_ctx = max_ctx; a.hq = num_q_heads; a.scale = scale;
    return q8::launch_decode(x, workspace, (hipStream_t)stream);
}

}  // extern "C"
