/*
 * ag_latent.h - a paged cache of latent vectors, and attention over it.
 *
 * Latent attention keeps ONE row a token that all query heads share: latent_dim channels that are key and value alike, and rope_dim channels that carry
 * the position and are key only.  In its absorbed form - the products that would expand a latent vector to every head's keys and values are folded
 * into the queries before and into the outputs after, by the caller - attention reads nothing but these rows:
 *     S[t,h,j] = scale * Q[t,h,:] . row[j],   O[t,h,:] = softmax_j(S) . row[j][0 .. latent_dim),   j <= position of t
 * with Q [T][H][latent_dim + rope_dim] (the latent part first) and O [T][H][latent_dim].  A token is latent_dim + rope_dim numbers whatever the
 * number of heads, so that a decode step of many heads is bound by the matrix units about as much as by memory.
 *
 * Conventions (pointers, streams, status codes, block tables, lengths, cu_new, order between append and attention, rows behind the last
 * session) are those of ag.h.  What differs:
 *   - pool  bf16 [num_pages][page_size][row], row = latent_dim + rope_dim rounded up to a multiple of 64 (ag_latent_row()); what is past
 *     latent_dim + rope_dim in a row is never written, and nothing depends on it.
 *   - Everything is bf16.  latent_dim 128, 256 or 512; rope_dim 32 or 64; page_size a power of two in [16, 256] (AG_ERR_UNSUPPORTED otherwise); any
 *     number of heads; all pointers 16-byte aligned (AG_ERR_INVALID_ARG otherwise).
 *   - max_ctx is at most 2^31 - 1025 (AG_ERR_INVALID_ARG beyond it).
 *   - Scores and the softmax's sums are fp32; softmax weights are rounded to bf16 for the value product, and summed as rounded.
 *   - Latent channels up to 2^60 in magnitude: a softmax weight stands at up to 2^40 (under the largest score of the first keys that a workgroup meets, not of all),
 *     so that fp32 sums of larger ones may come out infinite where the result is not.
 *   - Slots that no token uses may hold anything, NaN included.  Table entries that no token uses are not followed.
 *   - What is not finite in a row reaches the query rows that see its token, and no other.
 *   - Results are reproducible: partial results are merged in a fixed order, same inputs give the same bits (under
 *     the same total_new, max_new and max_ctx, on streams of as many CUs: these decide how a batch is cut).
 */
#ifndef AG_LATENT_H
#define AG_LATENT_H

#include "ag_rope.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Describes caller-owned device memory; plain data, read during the call only. */
typedef struct {
    void*   pool;              /* device, [num_pages][page_size][ag_latent_row(latent_dim, rope_dim)] bf16 */
    int32_t num_pages;
    int32_t page_size;
    int32_t latent_dim;
    int32_t rope_dim;
} ag_latent_cache;

/* Channels of a cache row; 0 for widths that no cache has. */
AG_API int32_t ag_latent_row(int32_t latent_dim, int32_t rope_dim);

/*
 * Append: new token i of session s (row cu_new[s] + i of latent_new and rope_new) is written to logical position prefix_lens[s] + i, its rotary part
 * rotated by that position on the way (rope: rot_dim = rope_dim; NULL copies rows that are rotated already).  latent_new is [T][latent_dim] and rope_new
 * [T][rope_dim], with token strides of their own in elements (multiples of 8): both may be slices of one projection's rows.
 * total_new >= cu_new[batch] sizes the launch, and both have so many rows: those behind the last session's may be read.
 */
AG_API ag_status ag_kv_append_latent(const ag_latent_cache* cache, const ag_rope* rope, const void* latent_new, int64_t latent_stride,
                              const void* rope_new, int64_t rope_stride,
                              const int32_t* block_tables, int32_t max_pages_per_seq,
                              const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                              int32_t batch, int32_t total_new, void* stream);

/*
 * Decode: one query a session and head over all ctx_lens[s] positions (the step's own token counted, and appended already); ctx_lens[s] = 0 gives
 * rows of zeros.  workspace_bytes >= ag_attn_decode_latent_workspace_bytes(batch, num_q_heads, latent_dim, max_ctx), 16-byte aligned, whose
 * previous contents do not matter; calls that share one must be ordered.
 */
AG_API size_t    ag_attn_decode_latent_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t latent_dim, int32_t max_ctx);
AG_API ag_status ag_attn_decode_latent(const ag_latent_cache* cache, const void* q, void* out,        /* device [B][H][..] */
                                const int32_t* block_tables, int32_t max_pages_per_seq,
                                const int32_t* ctx_lens,                               /* device [B] */
                                int32_t batch, int32_t max_ctx, int32_t num_q_heads, float scale,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * Resume prefill: row i of session s sits at position prefix_lens[s] + i and sees rows 0 .. prefix_lens[s] + i of the cache, the chunk's own
 * appended already.  With every prefix 0 it is the cold prefill.  max_new and max_ctx as for ag_attn_resume; the workspace as above, of
 * ag_attn_resume_latent_workspace_bytes(batch, total_new, num_q_heads, latent_dim, max_ctx) bytes.
 */
AG_API size_t    ag_attn_resume_latent_workspace_bytes(int32_t batch, int32_t total_new, int32_t num_q_heads, int32_t latent_dim, int32_t max_ctx);
AG_API ag_status ag_attn_resume_latent(const ag_latent_cache* cache, const void* q, void* out,        /* device [T][H][..] */
                                const int32_t* block_tables, int32_t max_pages_per_seq,
                                const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                                int32_t batch, int32_t total_new, int32_t max_new, int32_t max_ctx,
                                int32_t num_q_heads, float scale,
                                void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AG_LATENT_H */
