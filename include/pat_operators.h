/*
 * pat_operators.h -- C ABI of the operators of a layer that answers one prompt several times on 8-bit weights
 * (libpat_decode.so).
 *
 * What it is: reinforcement learning samples a group of answers to each prompt.  Their caches begin with the same keys
 * and values, so the decode step's attention needs to read those once per group, and the step's other bytes are
 * weights, which 8 bits halve.  Three operators, beside the single operators of pat_decode.h:
 *   - rotation of new tokens' q and k at their positions and the append of k and v to the paged cache;
 *   - decode attention in which the sequences of a group share the pages of a prefix;
 *   - y = x W^T with W in 8-bit floating point, a power-of-two scale per block of 128.
 *
 * Conventions are those of pat_decode.h's single operators: pointers are device memory of the CURRENT device, work is
 * enqueued on `hip_stream` and asynchronous, the library allocates nothing, every call returns PAT_OK or a negative
 * PAT_E* code and enqueues nothing on error.  Calls can be captured into a graph.  Activations have a type code; the
 * cache is bf16 in the layout of the decoder's pool: [n_pages][n_kv_heads][page_tokens][head_dim], K and V apart, one layer
 * (a layer's part of the decoder's own pool can be given), page_tokens in {16, 32, 64, 128}, head_dim in {64, 128}.
 * A page table has a row of max_pages page ids for each sequence: position p lies in page table[p / page_tokens].
 * Array contents live on the device, where no host check reaches them: what the kernels do with values out of range
 * is said at each call; none of it leaves the given buffers.
 */
#ifndef PAT_OPERATORS_H
#define PAT_OPERATORS_H

#include <stdint.h>
#include "pat_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PAT_F32  0
#define PAT_BF16 1

/* cos_sin[pos][j] = (cos, sin) of pos * base^(-2 j / head_dim), j < head_dim / 2, formed in 64 bits: float[n_pos][head_dim / 2][2],
 * 16-byte aligned, n_pos <= 2^25.  A program makes it once. */
int pat_op_rope_table(int64_t n_pos, int32_t head_dim, double base, float *cos_sin, void *hip_stream);

/* Row i of qkv [rows, ld] (ld elements from row to row) holds the n_q_heads q heads, then the n_kv_heads k heads, then the
 * v heads of the token of sequence seq[i] at position pos[i]: one row per sequence in a decode step, many where prompts are
 * prefilled, in any order.  With gains gq, gk (bf16 [head_dim], both or neither) each q and k head first gets an RMSNorm
 * with epsilon eps.  q and k heads are rotated: features (j, j + head_dim / 2) by the angle of (pos[i], j).  q goes to row i of
 * q_out [rows, ldq] in qkv's type (it may be qkv itself with ldq = ld; other overlaps are refused), k and v rounded to the cache.
 *   16-byte alignment: qkv, q_out, cos_sin, the pools, and ld and ldq in bytes.  rows * (heads of a row) < 2^28 (fp32 heads of 128 features: < 2^28 - 15).
 *   seq[i] < 0 is a row of padding: nothing is read or written for it.
 *   seq[i] >= n_seqs, pos[i] outside [0, n_pos) or the table's row, a page id outside [0, n_pages): nothing is written for the row,
 *   and *skipped (device, or NULL) is raised by one.
 *   Two rows that name the same position of a sequence leave one of their values, element by element, in its place. */
int pat_op_kv_append(const void *qkv, int32_t type, int64_t ld, int32_t rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                     const int32_t *seq, const int32_t *pos, const float *cos_sin, int32_t n_pos, const void *gq, const void *gk, float eps,
                     void *k_pages, void *v_pages, int32_t n_pages, int32_t page_tokens, const int32_t *page_table, int32_t n_seqs,
                     int32_t max_pages, void *q_out, int64_t ldq, int32_t *skipped, void *hip_stream);

/* Attention of one query token per sequence over its kv_len[s] cached tokens (the new one among them), where sequences
 * group_start[g] .. group_start[g + 1] - 1 are a group whose first shared_len[g] tokens are the same: their rows of the page
 * table name the same pages there (of a last page that the prefix fills in part each may have its own copy).
 * Keys [0, shared_len[g]) are read once, through one of the group's rows, for all of its sequences that are at least as long;
 * a shorter sequence is read through its own row.  shared_len[g] <= 0: the group shares nothing.  kv_len[s] = 0: no keys, the
 * result is zero (a slot of padding).
 *
 * pat_op_attn_plan cuts the step's work from the lengths on the device; its result serves every layer's pat_op_attn_shared
 * until a length changes.  group_start is int32[n_groups + 1] from 0 to n_seqs, ascending (equal values: an empty group);
 * n_seqs and n_groups 1 .. 2048 (a step without sequences has nothing to call).  plan: pat_op_attn_plan_bytes() bytes, 16-byte aligned.  A kv_len[s] below 0 or above max_len, or
 * group_start that is no such list, gives NaN as the result of the sequence, or of all, and so does a page id outside
 * [0, n_pages) or a length beyond max_pages, of the sequences that need the page.
 *
 * pat_op_attn_shared: q [n_seqs, ldq] and out [n_seqs, ldo], n_q_heads * head_dim used, of one type (out may be q itself with ldo = ldq); scores
 * q k / sqrt(head_dim); 16-byte alignment (q, out, pools, ldq and ldo in bytes); scratch pat_op_attn_scratch_bytes() bytes, 256-byte aligned,
 * overwritten, so calls that overlap in time need one each.  A plan is only read.  A sequence's result does not depend on
 * the values of keys behind its end.  A plan made for another n_seqs, n_q_heads or n_kv_heads gives NaN throughout. */
int64_t pat_op_attn_plan_bytes(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads);
int64_t pat_op_attn_scratch_bytes(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);
int pat_op_attn_plan(const int32_t *kv_len, const int32_t *group_start, const int32_t *shared_len, int32_t n_seqs, int32_t n_groups,
                     int32_t max_len, int32_t n_q_heads, int32_t n_kv_heads, void *plan, void *hip_stream);
int pat_op_attn_shared(const void *q, int32_t type, int64_t ldq, int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                       const void *k_pages, const void *v_pages, int32_t n_pages, int32_t page_tokens, const int32_t *page_table,
                       int32_t max_pages, const void *plan, void *out, int64_t ldo, void *scratch, void *hip_stream);

/* The 8-bit form of a block of numbers: 4 exponent and 3 mantissa bits (largest value 448, no infinity) times 2^e, e the
 * smallest integer with max|x| <= 448 2^e (0 for a block of zeros; not below -127), each element rounded to nearest even.
 * Elements that are not finite become NaN and do not count for the scale.  A weight's blocks are 128 rows by 128
 * columns, an activation's one row by 128 columns; the last ones of a row or column may be shorter.
 *
 * pat_op_f8_pack_weight brings w [n, k] (ld elements from row to row) into that form, once: packed (256-byte aligned)
 * pat_op_f8_weight_bytes() bytes, scales (4-byte aligned) pat_op_f8_scale_bytes() bytes.
 * pat_op_f8_gemm: y [m, ldy] = (mode 0) or += (mode 1) x W^T for x [m, ldx], both of any type code (m = 0 does nothing): x is
 * brought to its 8-bit form on the way, sums are fp32, the result is rounded once.  For an fp32 y the products are exact; for a
 * bf16 y the 8-bit matrix instruction forms them, which drops what lies far below the largest product of its group:
 * 5e-6 of a result row's norm for values of a normal distribution, 5e-5 for values of every exponent, where y's own rounding is 2e-3.
 * n <= 2^22, k <= 2^20, m <= 2^19, m n <= 2^36.  scratch: pat_op_f8_gemm_scratch_bytes() bytes, 256-byte aligned, overwritten.  y must not overlap x: such a call is refused. */
int64_t pat_op_f8_weight_bytes(int32_t n, int32_t k);
int64_t pat_op_f8_scale_bytes(int32_t n, int32_t k);
int pat_op_f8_pack_weight(const void *w, int32_t type, int64_t ld, int32_t n, int32_t k, void *packed, void *scales, void *hip_stream);
int64_t pat_op_f8_gemm_scratch_bytes(int32_t n, int32_t k, int32_t m);
/* The kernel that pat_op_f8_gemm launches (diagnostics, host only): plan[0] 0 the streaming product with x as it is, 1 the same after x was brought to its 8-bit
 * form, 2 the product by tiles (more than 64 rows); plan[1], plan[2] tiles of 16 rows of W and of x per workgroup, plan[3] its waves, plan[4] cuts of k.
 * Returns PAT_EINVAL for sizes or types that pat_op_f8_gemm refuses, and for m = 0. */
int pat_op_f8_gemm_plan(int32_t n, int32_t k, int32_t m, int32_t x_type, int32_t y_type, int32_t plan[5]);
int pat_op_f8_gemm(const void *w_packed, const void *w_scales, int32_t n, int32_t k, const void *x, int32_t x_type, int64_t ldx, int32_t m,
                   void *y, int32_t y_type, int64_t ldy, int32_t mode, void *scratch, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PAT_OPERATORS_H */
