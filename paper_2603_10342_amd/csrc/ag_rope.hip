// C-ABI entry points of rotary positions: argument validation, as ag_api.hip does it for the others (see include/ag_rope.h).
#include <math.h>

#include "rope_internal.h"

namespace ag {
namespace rope {

ag_status check(const ag_rope* r, int most)
{
    if (!r || !r->turns) { set_error("rope or its turns are NULL"); return AG_ERR_INVALID_ARG; }
    if ((uintptr_t)r->turns % 8) { set_error("turns must be 8-byte aligned"); return AG_ERR_INVALID_ARG; }
    if (r->rot_dim < 16 || r->rot_dim > 256 || r->rot_dim % 16) {
        set_error("rot_dim %d unsupported (multiple of 16, at most 256)", r->rot_dim);
        return AG_ERR_UNSUPPORTED;
    }
    if (r->rot_dim > most) { set_error("rot_dim %d exceeds the %d channels of a row", r->rot_dim, most); return AG_ERR_INVALID_ARG; }
    if (r->layout != AG_ROPE_HALVES && r->layout != AG_ROPE_PAIRS) { set_error("rope layout %d unsupported", r->layout); return AG_ERR_UNSUPPORTED; }
    if (!(r->magnitude > 0.0f) || !(r->magnitude < 1e30f)) { set_error("magnitude must be positive and finite"); return AG_ERR_INVALID_ARG; }
    return AG_OK;
}

namespace {

bool aligned(const void* p) { return (uintptr_t)p % 16 == 0; }

// Workgroups of a launch of 256 threads each: HIP refuses 2^32 threads along a dimension of the grid.
constexpr int64_t kMostWorkgroups = 0xFFFFFFFFll / 256;

ag_status check_lengths(const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new, int batch, int total)
{
    if (!prefix_lens || !new_lens || !cu_new) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if (batch <= 0 || total < 0) { set_error("batch=%d total_new=%d: sizes must be positive", batch, total); return AG_ERR_INVALID_ARG; }
    return AG_OK;
}

}  // namespace
}  // namespace rope
}  // namespace ag

using namespace ag;

extern "C" {

ag_status ag_rope_turns(double* turns, int32_t rot_dim, double base, int32_t scaling, double factor, double trained_len, double low, double high)
{
    if (!turns) { set_error("turns are NULL"); return AG_ERR_INVALID_ARG; }
    if (rot_dim < 2 || rot_dim % 2) { set_error("rot_dim %d is not a positive even number", rot_dim); return AG_ERR_INVALID_ARG; }
    if (!(base > 0) || !(base < INFINITY) || !(factor > 0) || !(factor < INFINITY)) { set_error("base and factor must be positive and finite"); return AG_ERR_INVALID_ARG; }
    if (scaling != AG_ROPE_PLAIN && scaling != AG_ROPE_LINEAR && scaling != AG_ROPE_RAMP) { set_error("rope scaling %d unsupported", scaling); return AG_ERR_UNSUPPORTED; }
    if (scaling == AG_ROPE_RAMP && (!(trained_len > 0) || !(trained_len < INFINITY) || !(low >= 0) || !(low < high) || !(high < INFINITY))) {
        set_error("a ramp needs trained_len > 0 and 0 <= low < high, all finite");
        return AG_ERR_INVALID_ARG;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double plain = pow(base, -2.0 * i / rot_dim) / 6.283185307179586477;
        double stays = scaling == AG_ROPE_PLAIN ? 1.0 : 0.0;          // the share that is not interpolated
        if (scaling == AG_ROPE_RAMP) stays = fmin(fmax((trained_len * plain - low) / (high - low), 0.0), 1.0);
        turns[i] = plain * (stays + (1.0 - stays) / factor);
    }
    return AG_OK;
}

ag_status ag_rope_rows(const ag_rope* rope, int32_t dtype, const void* x, int64_t x_token_stride, int64_t x_head_stride, void* y,
                       int64_t y_token_stride, int64_t y_head_stride, int32_t num_heads, int32_t head_dim, const int32_t* prefix_lens,
                       const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new, int32_t transposed, void* stream)
{
    if (dtype != AG_F32 && dtype != AG_BF16) { set_error("dtype %d unsupported", dtype); return AG_ERR_UNSUPPORTED; }
    if (head_dim <= 0 || head_dim % 8 || head_dim > 65536) { set_error("head_dim %d is not a positive multiple of 8, at most 65536", head_dim); return AG_ERR_INVALID_ARG; }
    ag_status st = rope::check(rope, head_dim);
    if (st) return st;
    if (!x || !y) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if ((st = rope::check_lengths(prefix_lens, new_lens, cu_new, batch, total_new))) return st;
    const rope::Units us(head_dim, rope->rot_dim / 2);
    if (num_heads <= 0 || (int64_t)num_heads * us.count() > 1 << 28) { set_error("num_heads=%d must be positive, and num_heads * head_dim at most 2^31", num_heads); return AG_ERR_INVALID_ARG; }
    const int64_t most = INT64_MAX >> 34, eight = dtype == AG_BF16 ? 8 : 4;          // (the last row's offset in bytes fits 64 bits)
    for (int64_t s : {x_token_stride, x_head_stride, y_token_stride, y_head_stride})
        if (s < 0 || s > most || s % eight) { set_error("strides must be multiples of 16 bytes and not negative"); return AG_ERR_INVALID_ARG; }
    if (!rope::aligned(x) || !rope::aligned(y)) { set_error("x and y must be 16-byte aligned"); return AG_ERR_INVALID_ARG; }
    if (x == y && (x_token_stride != y_token_stride || x_head_stride != y_head_stride)) { set_error("rows that are rotated where they stand have one pair of strides"); return AG_ERR_INVALID_ARG; }
    if ((total_new > 1 && y_token_stride < head_dim) || (num_heads > 1 && y_head_stride < head_dim)) {
        set_error("rows of y overlap each other: strides %lld and %lld of %d channels", (long long)y_token_stride, (long long)y_head_stride, head_dim);
        return AG_ERR_INVALID_ARG;
    }
    if (total_new == 0) return AG_OK;
    if ((total_new + 3ll) / 4 > rope::kMostWorkgroups) { set_error("total_new=%d: too many rows for one launch", total_new); return AG_ERR_INVALID_ARG; }
    return rope::launch_rows(rope::RowsArgs{rope::spec_of(*rope, transposed != 0), rope->layout, dtype, x, x_token_stride, x_head_stride, y, y_token_stride,
                                            y_head_stride, num_heads, head_dim, prefix_lens, new_lens, cu_new, batch, total_new}, (hipStream_t)stream);
}

ag_status ag_kv_append_rope(const ag_kv_cache* cache, const ag_rope* rope, const void* q, void* q_out, int32_t num_q_heads, const void* k_new,
                            const void* v_new, const int32_t* block_tables, int32_t max_pages_per_seq, const int32_t* prefix_lens,
                            const int32_t* new_lens, const int32_t* cu_new, int32_t batch, int32_t total_new, void* stream)
{
    CacheView c;
    ag_status st = view_cache(cache, &c);
    if (st) return st;
    if (c.ps < 16) { set_error("page_size %d unsupported by the rotating append (16 or more)", c.ps); return AG_ERR_UNSUPPORTED; }
    if ((st = rope::check(rope, c.d))) return st;
    if (!k_new || !v_new || !block_tables || !q != !q_out) { set_error("a required pointer is NULL"); return AG_ERR_INVALID_ARG; }
    if ((st = rope::check_lengths(prefix_lens, new_lens, cu_new, batch, total_new))) return st;
    if (max_pages_per_seq <= 0) { set_error("max_pages_per_seq=%d must be positive", max_pages_per_seq); return AG_ERR_INVALID_ARG; }
    if (q ? num_q_heads <= 0 || num_q_heads % c.hkv || num_q_heads / c.hkv > 1 << 16 : num_q_heads != 0) {
        set_error("num_q_heads %d is not a positive multiple of num_kv_heads %d, at most 65536 of them (0 without q)", num_q_heads, c.hkv);
        return AG_ERR_INVALID_ARG;
    }
    if (!rope::aligned(k_new) || !rope::aligned(v_new) || !rope::aligned(q) || !rope::aligned(q_out) || !rope::aligned(c.k) || !rope::aligned(c.v)) {
        set_error("q, q_out, k_new, v_new and the pools must be 16-byte aligned");
        return AG_ERR_INVALID_ARG;
    }
    if (total_new == 0) return AG_OK;
    if (total_new / 16 + 2ll * batch > rope::kMostWorkgroups || c.hkv > 65535) { set_error("too many groups or heads for one launch"); return AG_ERR_INVALID_ARG; }
    return rope::launch_append(rope::AppendArgs{c, rope::spec_of(*rope), rope->layout, q, q_out, num_q_heads, k_new, v_new, block_tables, max_pages_per_seq,
                                                prefix_lens, new_lens, cu_new, batch, total_new}, (hipStream_t)stream);
}

}  // extern "C"
