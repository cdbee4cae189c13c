/*
 * kb_attention.h -- the operators of an attention block whose outputs the gate judges, for serving: norms
 * of queries and keys with the position rotation, attention over whole prompts, attention of one new
 * token over a paged cache.
 *
 * The gate's third workload is modelled on an attention output of 32 heads of 128; these calls make such outputs
 * and a baseline kernel to compare candidates' times with.  (Attention is also one of the workloads whose kernels the
 * paper searches, SDPAttn in Appendix "Benchmark Descriptions and Shapes", with heads of 1024: those are beyond
 * KB_ATTENTION_MAX_DIM and are refused.)  The conventions of kb.h and kb_ops.h hold.  They are a serving
 * path's forms: no call here has a gradient.  In addition:
 *   - Heads of a packed batch are [tokens][heads][dim]: the elements of dim are adjacent, and the
 *     strides between tokens (..._row) and heads (..._head) are free, in elements.  Slices of one
 *     projection [tokens][(q_heads + 2 kv_heads) dim] are such tensors.
 *   - Query head h reads key and value head h / (q_heads / kv_heads); q_heads is a multiple of kv_heads.
 *   - Numbers that only the device knows (offsets, lengths, pages, slots) are checked there: nothing is
 *     read or written out of range, and the device status (kb_ctx_poll) becomes KB_ERR_INVALID_ARG.
 */
#ifndef KB_ATTENTION_H_
#define KB_ATTENTION_H_

#include "kb_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest dim of a head: of the attention calls, and of kb_qk_norm_rope. */
#define KB_ATTENTION_MAX_DIM 128u
#define KB_ROPE_MAX_DIM 256u

/* Keys and values by pages: element d of head h of slot s (0 <= s < pages * page_size) is at
 *     d_k + (s / page_size) * k_page + (s % page_size) * k_row + h * k_head + d
 * and likewise for the values; strides in elements, any order of the axes. */
typedef struct {
  void* d_k;
  void* d_v;
  uint64_t k_page, k_row, k_head;
  uint64_t v_page, v_row, v_head;
  uint64_t pages;     /* pages * page_size at most 2^31 - 1 */
  uint32_t page_size; /* >= 1 */
} kb_paged_cache;

/* ---- norms and rotation of queries and keys ------------------------------------------------
 *
 * Per token t and head of q and of k, in binary32, x its dim elements:
 *     x = x / sqrt(sum(x^2) / dim + eps) * weight                         (norm = 1; left out with norm = 0)
 *     a' = a cos(w) - b sin(w),  b' = b cos(w) + a sin(w)      w = position[t] * inv_freq[i]
 * for the pairs (a, b) = (x[i], x[i + r/2]), or (x[2i], x[2i + 1]) with interleaved = 1, i < r/2 and
 * r = rotary_dim; the elements from r on are not turned.  The angle is reduced to a part of a turn
 * before it is rounded: beside that rounding it is off by at most 2^-63 turns times the position (and 2^-74 inv_freq
 * turns times the position), which is nothing up to positions of 2^36 on either side of 0.
 *
 *   d_q, d_k         DEVICE heads of `dtype` (KB_F32, KB_F16 or KB_BF16); dim 1 .. 256.
 *   norm, eps        eps is finite and > 0 with norm = 1 and not looked at with norm = 0.
 *   d_q_weight, d_k_weight  DEVICE [dim] of `param_dtype` (`dtype` or KB_F32); NULL: 1.
 *   d_positions      DEVICE [tokens], any 64-bit number (how near far ones come: above).
 *   d_inv_freq       DEVICE [r/2] binary64, radians per position, finite; NULL with r = 0.
 *   rotary_dim       even, 0 .. dim.
 *   d_q_out          DEVICE heads, or NULL.  May be d_q itself, with the same strides.
 *   d_k_out          the same for the keys.
 *   cache, d_slots   NULL, or where the turned keys and the values d_v go as well: DEVICE [tokens] slots;
 *                    a negative one stores nothing.  Each slot comes once; in one that comes twice
 *                    the elements are one token's or the other's, each by itself.  Slots and heads of the
 *                    cache do not overlap (strides that let them are refused).
 *   d_v              DEVICE heads of the values; NULL without a cache.
 * At least one of d_q_out, d_k_out and cache is not NULL. */
kb_status kb_qk_norm_rope(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                          const void* d_k, uint64_t k_row, uint64_t k_head, uint32_t kv_heads, uint64_t tokens,
                          uint32_t dim, kb_dtype dtype, int norm, const void* d_q_weight, const void* d_k_weight,
                          kb_dtype param_dtype, float eps, const int64_t* d_positions, const double* d_inv_freq,
                          uint32_t rotary_dim, int interleaved, void* d_q_out, uint64_t q_out_row,
                          uint64_t q_out_head, void* d_k_out, uint64_t k_out_row, uint64_t k_out_head,
                          const void* d_v, uint64_t v_row, uint64_t v_head, const kb_paged_cache* cache,
                          const int64_t* d_slots, void* stream);

/* ---- attention over whole prompts ------------------------------------------------------------
 *
 * Sequence s has the queries q_offsets[s] .. q_offsets[s + 1] - 1 (nq of them) and the keys
 * k_offsets[s] .. k_offsets[s + 1] - 1 (nk).  Its query i sees the keys j with j - i <= nk - nq (causal = 1:
 * the last query sees all) or all (causal = 0).  Per query and head, over the keys it sees:
 *     s_j = scale * sum_d q[d] k_j[d];   lse = log sum_j exp(s_j);   out = sum_j exp(s_j - lse) v_j
 * Products of 16-bit numbers are added in binary32 on the tensor cores, exponentials and their sum are
 * binary32, and exp(s_j - ...) is rounded to `dtype` (relative to a running largest value) before it
 * meets v_j; out is rounded once.  (The largest exponential of a query is between 2^7 and 2^15 there, so that bfloat16
 * values of 2^112 and more, over the number of keys, can make a sum infinite.  A score of 2^24 or more in magnitude has no
 * digits behind the point in binary32: what comes of such scores is not defined.)  A query with no score above -infinity (none at all, above all) has
 * out = 0 and lse = -infinity.  Keys and values that a query does not see do not touch its outputs, whatever
 * they hold; a value that is not finite makes that element of the queries that see it infinite or NaN.
 *
 *   d_q              DEVICE heads of `dtype` (KB_F16 or KB_BF16), q_tokens of them.
 *   d_k, d_v         DEVICE heads, k_tokens of them.  Pointers of q, k and v 16-byte aligned, row and head
 *                    strides multiples of 8, not 0, less than 2^39; dim a multiple of 8 up to 128.
 *   d_q_offsets, d_k_offsets  DEVICE [sequences + 1], ascending, within 0 .. q_tokens (k_tokens); both
 *                    NULL for one sequence of all tokens.  Queries outside every sequence are not written.
 *   sequences        at most 2^24, of at most 2^24 keys each.
 *   scale            > 0, at most 2^127.
 *   d_out            DEVICE heads of `dtype`; does not overlap the inputs.
 *   d_lse            DEVICE binary32 [q_tokens][q_heads]; NULL: not written. */
kb_status kb_attention(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                       uint64_t q_tokens, const void* d_k, uint64_t k_row, uint64_t k_head, const void* d_v,
                       uint64_t v_row, uint64_t v_head, uint32_t kv_heads, uint64_t k_tokens, uint32_t dim,
                       kb_dtype dtype, const int32_t* d_q_offsets, const int32_t* d_k_offsets, uint32_t sequences,
                       int causal, float scale, void* d_out, uint64_t out_row, uint64_t out_head, float* d_lse,
                       void* stream);

/* ---- attention of one new token over a paged cache ---------------------------------------------
 *
 * The same formulas for one query per sequence, which sees the first lengths[s] slots of its pages: key j
 * of sequence s is in slot table[s][j / page_size] * page_size + j % page_size of the cache.
 *
 *   d_q              DEVICE heads [sequences][q_heads][dim] of `dtype` (KB_F16 or KB_BF16).
 *   cache            pointers 16-byte aligned, strides multiples of 8, not 0, less than 2^39; dim a multiple
 *                    of 8 up to 128.
 *   d_table          DEVICE [sequences][max_pages], row stride table_row; entries past a sequence's last
 *                    page are not looked at.
 *   d_lengths        DEVICE [sequences], 0 .. max_pages * page_size (the new token's own key included);
 *                    sequences * max_pages * page_size at most 2^36.
 *   d_out, d_lse     DEVICE heads [sequences][q_heads][dim]; binary32 [sequences][q_heads] or NULL.
 * Keys on a page outside the cache, or past max_pages, are left out.  Long sequences are divided over
 * the card; the parts meet in a workspace of the context whose size no call changes: the first call
 * outside a capture allocates it, or kb_attention_paged_reserve.  The division follows from the
 * lengths and the card alone, and so do the sums' orders. */
kb_status kb_attention_paged(kb_ctx* ctx, const void* d_q, uint64_t q_row, uint64_t q_head, uint32_t q_heads,
                             const kb_paged_cache* cache, uint32_t kv_heads, uint32_t dim, kb_dtype dtype,
                             const int32_t* d_table, uint64_t table_row, uint32_t max_pages,
                             const int32_t* d_lengths, uint32_t sequences, float scale, void* d_out,
                             uint64_t out_row, uint64_t out_head, float* d_lse, void* stream);

/* The workspace, for calls that are then captured into a graph (a capture cannot allocate it).
 * `stream` is only asked whether it is being captured. */
kb_status kb_attention_paged_reserve(kb_ctx* ctx, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KB_ATTENTION_H_ */
