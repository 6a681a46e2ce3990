/*
 * ag_q8.h - the paged KV cache in 8 bits, and attention over it.
 *
 * The same request classes as ag.h (cold prefill, resume prefill, short decode, append) over a cache that holds keys and
 * values as e4m3 numbers: half the bytes of bf16, which is what a decode step is bound by, and twice the tokens in a pool.
 * Every (token, KV head) row of keys and of values has a power of two of its own, found when the row is appended, so that
 * nothing has to be calibrated and a token's row never changes once it is written:
 *     e  = the least exponent with max |x| <= 448 * 2^e over the row's finite entries, kept in [-110, 119], stored as the byte e + 127
 *     x8 = e4m3(x * 2^-e), to nearest, ties to even; what is not finite is stored as NaN
 *     x^ = x8 * 2^e, which is what attention reads (a bf16 number, exactly)
 * An entry is off by at most 2^-4 of itself, or 2^-10 * 2^e where that is more (2^-17 of the row's largest, unless e is
 * at its lowest).  Rows of zeros are stored as zeros.  Magnitudes above 448 * 2^119 (0.875 of bf16's and fp32's range) are stored as that.
 *
 * Conventions (pointers, streams, status codes, block tables, lengths, cu_new, GQA, order between append and attention) are
 * those of ag.h.  What differs:
 *   - `dtype` is the type of the activations: of q, out, k_new, v_new, and of the rows that come back.
 *   - Layouts, 16-byte aligned (row-major, innermost last):
 *       K pool  e4m3  [num_pages][Hkv][page_size/4][D/16][4][16]   four slots of 16 channels: 64 bytes in a run
 *       V pool  e4m3  [num_pages][Hkv][page_size/16][D][16]        16 slots of a channel in a run
 *       exps    uint8 [num_pages][Hkv][2][page_size]               the exponent bytes of keys, then of values.  In each group of 16
 *                     slots the byte of slot s stands at 4 * (s % 4) + s / 4 for keys, at s for values.
 *   - Supported: AG_F32 and AG_BF16; head_dim a multiple of 16, <= 256; page_size a power of two in [16, 256]; any group size;
 *     q, out, k_new, v_new, k_out, v_out, the pools and exps 16-byte aligned (AG_ERR_INVALID_ARG otherwise).
 *   - max_ctx is at most 2^31 - 1025 (AG_ERR_INVALID_ARG beyond it).
 *   - Slots that no token uses may hold anything, NaN included: they are read, but nothing depends on them.  Table entries that no token uses are not followed.
 *     (ag_debug_validate looks at tables and lengths only: it takes an ag_kv_cache of the same num_pages, page_size, num_kv_heads, head_dim and dtype.)
 *   - fp32 activations keep 24 bits of queries and softmax weights in the products, as three bf16 terms, in every call.  bf16 activations: decode
 *     keeps them too, but with head_dim 128, page_size 16 and up to 16 heads a group, where weights are rounded to bf16 as over a bf16 cache of that
 *     shape; prefill and resume round them at every shape (over bf16 caches at that one only): off by up to 2^-8 of themselves, each for itself, beside
 *     cached values that are off by up to 2^-4 and an output rounded by up to 2^-8.  The pools do not depend on `dtype`: whoever wants all bits of the
 *     weights in prefill describes the same pools as AG_F32 and passes fp32 rows.
 *   - What is not finite in a key or a value reaches the rows that see its token, a value's in its own channel only, and no other row.
 *   - Scores are summed up in fp32 before `scale`, and attention divides by the sum of its weights at the end.  The accuracy above holds whatever the
 *     context for queries, keys and values whose rows' largest entries lie between 2^-60 and 2^80, a scale up to 2^60, and scores that fit: head_dim *
 *     max |q| * max |k| below 2^127, and so that times scale * log2 e.  Below these, last bits may be lost; above, sums may overflow and rows become NaN.
 */
#ifndef AG_Q8_H
#define AG_Q8_H

#include "ag.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Describes caller-owned device memory; plain data, read during the call only. */
typedef struct {
    void*   k_pool;            /* device, see above */
    void*   v_pool;
    void*   exps;
    int32_t num_pages;
    int32_t page_size;
    int32_t num_kv_heads;
    int32_t head_dim;
    int32_t dtype;             /* ag_dtype of the activations */
} ag_kv_cache_q8;

/*
 * ag_kv_append into an 8-bit cache: new token i of session s (row cu_new[s] + i of k_new / v_new) is quantised, as above, into
 * logical position prefix_lens[s] + i of every KV head.  The bytes are determined by the row alone.  Nothing but the new tokens'
 * own slots is written.  total_new >= cu_new[batch] sizes the launch; rows behind the last session's are nobody's.
 */
AG_API ag_status ag_kv_append_q8(const ag_kv_cache_q8* cache, const void* k_new, const void* v_new,   /* device [T][Hkv][D] */
                          const int32_t* block_tables, int32_t max_pages_per_seq,
                          const int32_t* prefix_lens, const int32_t* new_lens,   /* device [B] */
                          const int32_t* cu_new,                                 /* device [B+1] */
                          int32_t batch, int32_t total_new, void* stream);

/*
 * The way back: positions prefix_lens[s] .. prefix_lens[s] + new_lens[s] - 1 of session s as rows cu_new[s] .. of k_out and v_out,
 * x^ in the activations' type (exactly: both hold every such number).  Appending these rows to an 8-bit cache again gives values
 * that read back the same.  Rows behind the last session's are left as they were.
 */
AG_API ag_status ag_kv_read_q8(const ag_kv_cache_q8* cache, void* k_out, void* v_out,                 /* device [T][Hkv][D] */
                        const int32_t* block_tables, int32_t max_pages_per_seq,
                        const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                        int32_t batch, int32_t total_new, void* stream);

/* ag_attn_prefill over an 8-bit cache: causal attention of whole prompts, already appended. */
AG_API ag_status ag_attn_prefill_q8(const ag_kv_cache_q8* cache, const void* q, void* out,            /* device [T][Hq][D] */
                             const int32_t* block_tables, int32_t max_pages_per_seq,
                             const int32_t* new_lens, const int32_t* cu_new,
                             int32_t batch, int32_t total_new, int32_t max_new,
                             int32_t num_q_heads, float scale, void* stream);

/* ag_attn_resume over an 8-bit cache: row i of session s sees keys 0 .. prefix_lens[s] + i.  max_ctx and max_new as there. */
AG_API ag_status ag_attn_resume_q8(const ag_kv_cache_q8* cache, const void* q, void* out,             /* device [T][Hq][D] */
                            const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                            int32_t batch, int32_t total_new, int32_t max_new, int32_t max_ctx,
                            int32_t num_q_heads, float scale, void* stream);

/*
 * ag_attn_decode over an 8-bit cache: one query per session over all ctx_lens[s] positions; ctx_lens[s] = 0 gives a row of zeros.
 * workspace_bytes >= ag_attn_decode_q8_workspace_bytes(batch, num_q_heads, head_dim, max_ctx), 16-byte aligned, whose previous
 * contents do not matter; calls that share one must be ordered.  Partial results are merged in a fixed order: same inputs, same bits.
 */
AG_API size_t    ag_attn_decode_q8_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t head_dim, int32_t max_ctx);
AG_API ag_status ag_attn_decode_q8(const ag_kv_cache_q8* cache, const void* q, void* out,             /* device [B][Hq][D] */
                            const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* ctx_lens,                               /* device [B] */
                            int32_t batch, int32_t max_ctx,
                            int32_t num_q_heads, float scale,
                            void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AG_Q8_H */
