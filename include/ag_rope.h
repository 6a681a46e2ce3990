/*
 * ag_rope.h - rotary positions: rows rotated by their position, and the KV append that rotates on its way.
 *
 * The first rot_dim channels of a row at logical position p are pairs (a, b), pair i < rot_dim / 2 turned by the angle 2 pi p turns[i]:
 *     a' = m (a cos - b sin)      b' = m (b cos + a sin)
 * Channels rot_dim and up stay as they are.  Which channels make a pair is the layout's; m is the magnitude (1 unless a context's
 * scaling asks for another).  turns[i] are turns a position, in 64 bits, so that far positions keep their angles: frequency / (2 pi).
 *
 * Conventions (pointers, streams, status codes, block tables, lengths, cu_new, rows behind the last session) are those of ag.h.  What is rotated
 * keeps its type; a rotation is computed in fp32 from a cosine and a sine rounded to fp32, and rounded once.
 */
#ifndef AG_ROPE_H
#define AG_ROPE_H

#include "ag.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    AG_ROPE_HALVES = 0,        /* pair i is channels i and i + rot_dim / 2 */
    AG_ROPE_PAIRS = 1          /* pair i is channels 2 i and 2 i + 1 */
} ag_rope_layout;

/* Plain data, read during the call only. */
typedef struct {
    const double* turns;       /* device, [rot_dim / 2] */
    int32_t rot_dim;           /* a multiple of 16, from 16 to 256 */
    int32_t layout;            /* ag_rope_layout */
    float   magnitude;         /* m, positive and finite */
} ag_rope;

/*
 * Fills turns (HOST, [rot_dim / 2]) with base^(-2 i / rot_dim) / (2 pi), divided for contexts `factor` times the trained one as `scaling` says:
 *   AG_ROPE_PLAIN   not at all
 *   AG_ROPE_LINEAR  by factor: positions are interpolated
 *   AG_ROPE_RAMP    by a blend of the two, by how many turns r = trained_len * turns[i] a pair takes over the trained context: pairs of r <= low are
 *                   interpolated, those of r >= high stay, and between them turns are mixed in proportion g = (r - low) / (high - low):
 *                   turns * (g + (1 - g) / factor)
 * (A scaling by a larger base is base * factor^(rot_dim / (rot_dim - 2)).  Any other one is the caller's own array.)
 * base and factor positive; trained_len, low and high are read by AG_ROPE_RAMP only: trained_len > 0, 0 <= low < high.
 */
typedef enum { AG_ROPE_PLAIN = 0, AG_ROPE_LINEAR = 1, AG_ROPE_RAMP = 2 } ag_rope_scaling;
AG_API ag_status ag_rope_turns(double* turns, int32_t rot_dim, double base, int32_t scaling, double factor, double trained_len, double low,
                        double high);

/*
 * Rotates rows: row cu_new[s] + i of x, head h, is at position prefix_lens[s] + i and goes to the same row and head of y.  x and y are
 * [T][heads][head_dim] with strides of their own in elements, channels contiguous: a slice of a wider row is rotated where it stands.
 * y may be x (same pointer, same strides); otherwise they may not overlap.  Rows of y may not overlap each other: its strides are head_dim or more where there are
 * more rows or heads than one (AG_ERR_INVALID_ARG otherwise); those of x may, and may be 0, where y is not x.  transposed != 0 applies the transposed matrix, sin with the other sign: the
 * rotation's gradient (m and all), and with m = 1 its inverse.  total_new >= cu_new[batch] sizes the launch, and x has so many rows: those behind the last
 * session's may be read; y's are left as they were.
 * head_dim a multiple of 8 and at least rot_dim; pointers 16-byte aligned and strides multiples of 16 bytes (AG_ERR_INVALID_ARG otherwise).
 */
AG_API ag_status ag_rope_rows(const ag_rope* rope, int32_t dtype, const void* x, int64_t x_token_stride, int64_t x_head_stride, void* y,
                       int64_t y_token_stride, int64_t y_head_stride, int32_t num_heads, int32_t head_dim,
                       const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                       int32_t batch, int32_t total_new, int32_t transposed, void* stream);

/*
 * ag_kv_append with the rotation on the way: keys go into their pages rotated, values as they are; and the same tokens' queries are rotated from q
 * into q_out in the same launch (q_out may be q; both NULL with num_q_heads = 0: no queries).  k_new is left as it was.  The pools and q_out hold
 * exactly what ag_rope_rows of k_new and q, and ag_kv_append of the rotated keys, would have put there.
 * (Over an 8-bit cache: ag_rope_rows, then ag_kv_append_q8 of ag_q8.h.)
 * page_size 16 or more (AG_ERR_UNSUPPORTED below); rot_dim at most head_dim; num_q_heads a multiple of num_kv_heads; all pointers 16-byte aligned.
 */
AG_API ag_status ag_kv_append_rope(const ag_kv_cache* cache, const ag_rope* rope,
                            const void* q, void* q_out, int32_t num_q_heads,              /* device [T][Hq][D] */
                            const void* k_new, const void* v_new,                         /* device [T][Hkv][D] */
                            const int32_t* block_tables, int32_t max_pages_per_seq,
                            const int32_t* prefix_lens, const int32_t* new_lens, const int32_t* cu_new,
                            int32_t batch, int32_t total_new, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AG_ROPE_H */
