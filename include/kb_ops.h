/*
 * kb_ops.h -- operators of large language models whose outputs the gate judges: layer norm
 * (forward, backward), quantisation to 8-bit floating point in blocks of 128, and the matrix
 * product of two such operands.
 *
 * The paper searches kernels for operators of models (Appendix "Benchmark Descriptions and Shapes":
 * RMSNorm, LinearReLUDiv, attention and others; none of those is here).  The calls of kb.h compare and
 * rank candidates; these calls make, in the gate's own storage types, the operands and a baseline kernel
 * for candidates of a linear layer in 8 bits.  They compute what they are asked for and nothing else:
 * gradients come from the backward calls, not from a framework's bookkeeping.
 *
 * The conventions of kb.h hold: plain C99 types, caller-owned buffers, work enqueued on
 * `stream` without synchronising, argument errors before any launch, one context per stream
 * and host thread at a time.  Every output is a pure function of the inputs (sums have a fixed
 * order).  In addition:
 *   - Matrices are row-major.  A leading dimension (ld...) counts elements and is at least the
 *     number of columns; the gap between rows is not written and what it holds does not matter.
 *   - Zero rows are allowed: nothing is written, except that sums over no row are zero.
 *   - Inputs and outputs of one call do not overlap.
 *   - Pointers need their element type's alignment; 16-byte aligned pointers and rows are
 *     faster.  Where more is needed, the call says so and refuses with KB_ERR_ALIGNMENT.
 *   - NaN and Inf are ordinary inputs: they reach the outputs that depend on them, no others.
 */
#ifndef KB_OPS_H_
#define KB_OPS_H_

#include "kb.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Elements along the contraction that share one scale. */
#define KB_BLOCK 128u
/* Limits checked at the boundary. */
#define KB_OPS_MAX_DIM 1073741824ull /* rows and columns of a matrix (2^30) */

typedef enum {
  KB_SCALE_ROWS = 0, /* one scale per row and block of 128 columns (1 x 128)            */
  KB_SCALE_TILES = 1 /* one scale per 128 rows and 128 columns (128 x 128)              */
} kb_scale_mode;

/* ---- block quantisation ----------------------------------------------------------------
 *
 * A matrix V [R][C] is stored as 8-bit codes Q [R][C] and binary32 scales S with
 *     V[r][c] ~ Q[r][c] * S[c / 128][r]          KB_SCALE_ROWS,   S is [ceil(C/128)][R]
 *     V[r][c] ~ Q[r][c] * S[c / 128][r / 128]    KB_SCALE_TILES,  S is [ceil(C/128)][ceil(R/128)]
 * Per block, every operation rounded to binary32 once, F = 448 (KB_F8E4M3) or 57344 (KB_F8E5M2):
 *     a = max(2^-100, largest |V| that is finite);  S = a / F
 *     Q = round((V * L * 0.875) / (a * L * (0.875 / F)))     = V * F / a, its quotient rounded once before
 * with round-to-nearest-even to the format.  0.875 / F is a power of two; L = 2^40 for a < 2^-60 and 1
 * elsewhere keeps the steps above binary32's smallest numbers.  NaN and +-Inf become the format's NaN and
 * do not enter a.
 *
 *   d_x        DEVICE [rows][cols] of `dtype` (KB_F32, KB_F16 or KB_BF16), row stride ldx.
 *   transpose  0: V = x (R = rows, C = cols).  1: V = the transpose of x (R = cols, C = rows):
 *              what a product that contracts over the rows of x takes.
 *   d_q        DEVICE [R][C] codes, row stride ldq (a multiple of 16 suits kb_matmul_blocks).
 *   d_scale    DEVICE binary32, contiguous, as above. */
kb_status kb_quantize_blocks(kb_ctx* ctx, const void* d_x, uint64_t rows, uint64_t cols, uint64_t ldx,
                             kb_dtype dtype, int transpose, kb_scale_mode mode, void* d_q, uint64_t ldq,
                             kb_dtype q_dtype, float* d_scale, void* stream);

/* ---- layer norm -------------------------------------------------------------------------
 *
 * Per row of n = cols elements, in binary32 (sums included):
 *     mean = sum(x) / n;  var = sum((x - mean)^2) / n;  rstd = 1 / sqrt(var + eps)
 *     y = (x - mean) * rstd * weight + bias
 *
 *   d_x              DEVICE [rows][cols] of `dtype` (KB_F32, KB_F16 or KB_BF16), row stride ldx.
 *   d_weight, d_bias DEVICE [cols] of `param_dtype` (`dtype` or KB_F32); NULL: 1 and 0.
 *   eps              finite and > 0.
 *   d_y              DEVICE [rows][cols] of `dtype`, row stride ldy; NULL: not written.
 *   d_mean, d_rstd   DEVICE binary32 [rows]; NULL: not written.
 *   d_q, d_scale     the binary32 y (before its rounding to `dtype`) quantised as by
 *                    kb_quantize_blocks with KB_SCALE_ROWS: DEVICE codes [rows][cols] with row
 *                    stride ldq in `q_dtype`, and DEVICE scales [ceil(cols/128)][rows].  Both
 *                    or neither NULL.
 * At least one output is not NULL.  cols >= 1. */
kb_status kb_layernorm(kb_ctx* ctx, const void* d_x, uint64_t rows, uint64_t cols, uint64_t ldx,
                       kb_dtype dtype, const void* d_weight, const void* d_bias, kb_dtype param_dtype,
                       float eps, void* d_y, uint64_t ldy, float* d_mean, float* d_rstd, void* d_q,
                       uint64_t ldq, kb_dtype q_dtype, float* d_scale, void* stream);

/* Its gradients.  With xh = (x - mean) * rstd and g = dy * weight, in binary32:
 *     dx = rstd * (g - sum(g)/n - xh * sum(g * xh)/n)      per row
 *     dweight = sum over rows of dy * xh,   dbias = sum over rows of dy
 *   d_dy, d_x        DEVICE [rows][cols] of `dtype`, row strides lddy and ldx.
 *   d_weight         as in the forward pass; NULL: 1.
 *   d_mean, d_rstd   DEVICE binary32 [rows], what the forward pass wrote.
 *   d_dx             DEVICE [rows][cols] of `dtype`, row stride lddx; NULL: not written.
 *   d_dweight, d_dbias  DEVICE [cols] of `param_dtype`; NULL: not written.
 * At least one output is not NULL.  Partial sums over rows live in the context's workspace, which
 * grows on demand.  A call that is captured into a graph uses the workspace as it is: it is refused with
 * KB_ERR_WORKSPACE if that would have to grow (kb_layernorm_backward_reserve, or such a call outside the
 * capture, makes room first).  Later growth leaves what a graph uses in place; a graph must not run after
 * the context is destroyed, nor at the same time as another call or graph on the context. */
kb_status kb_layernorm_backward(kb_ctx* ctx, const void* d_dy, uint64_t lddy, const void* d_x,
                                uint64_t ldx, uint64_t rows, uint64_t cols, kb_dtype dtype,
                                const void* d_weight, kb_dtype param_dtype, const float* d_mean,
                                const float* d_rstd, void* d_dx, uint64_t lddx, void* d_dweight,
                                void* d_dbias, void* stream);

/* Room for backward passes over at most `rows` rows of `cols` columns, whatever their types and strides.
 * `stream` is only asked whether it is being captured (then the call is refused where it would allocate). */
kb_status kb_layernorm_backward_reserve(kb_ctx* ctx, uint64_t rows, uint64_t cols, void* stream);

/* ---- product of two block-quantised matrices ---------------------------------------------
 *
 *     D[m][n] = sum over blocks kb of  SA[kb][m] * SB[kb][n or n/128] * sum_{k in kb} A[m][k] * B[n][k]
 * The inner sums run on the tensor cores in binary32; they are scaled and added in binary32, in
 * an order that the sizes alone fix, and D is rounded once.  Finite scales overflow or underflow only
 * where a block's part of D does, not in their own product (rows of a large product with tile scales in which
 * that product leaves binary32 are computed twice, the second time far slower).
 *
 *   d_a, d_b     DEVICE codes A [M][K] and B [N][K] (KB_F8E4M3 or KB_F8E5M2 each), row strides
 *                lda and ldb; pointers 16-byte aligned, strides multiples of 16.
 *   d_a_scale    DEVICE binary32 [ceil(K/128)][M] (KB_SCALE_ROWS).
 *   d_b_scale    DEVICE binary32 as kb_quantize_blocks lays it out for b_mode.
 *   d_d          DEVICE [M][N] of d_dtype (KB_F32, KB_F16 or KB_BF16), row stride ldd.
 * A linear layer y = x W^T takes A = x (rows), B = W (tiles); its input gradient dx = dy W takes
 * A = dy, B = the transpose of W (tiles); its weight gradient dW = dy^T x takes A and B = the
 * transposes of dy and x (rows).  M = 0 or N = 0: nothing to do; K = 0: D = 0. */
kb_status kb_matmul_blocks(kb_ctx* ctx, const void* d_a, uint64_t lda, kb_dtype a_dtype,
                           const float* d_a_scale, const void* d_b, uint64_t ldb, kb_dtype b_dtype,
                           const float* d_b_scale, kb_scale_mode b_mode, uint64_t M, uint64_t N,
                           uint64_t K, void* d_d, uint64_t ldd, kb_dtype d_dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KB_OPS_H_ */
