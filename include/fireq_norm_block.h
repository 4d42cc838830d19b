/*
 * fireq_norm_block.h -- the residual stream between two blocks that have a norm on both sides: the norm of a block's output, its gate and
 * factor, the residual's addition, and the norm in front of the next layer.
 *
 *   p[m,k] = X[m,k] * post[k] / sqrt( (1/K) sum_k X[m,k]^2 + eps )        (post_bf16 == NULL: p = X)
 *   H[m,k] = bf16( R[m,k] + scale * gate[g(m),k] * p[m,k] )               (gate_bf16 == NULL: 1)
 *   y[m,k] = H[m,k] * w[k] / sqrt( (1/K) sum_k H[m,k]^2 + eps )
 *
 * g(m) = gate_rows[m] where that is given; otherwise 0 where gates is 1 (a gate for all rows), and m where gates is M.  Sums, p and y are FP32;
 * H is rounded once, y is that of the rounded H.
 *
 *   fq_rmsnorm_block           Y_bf16[m,k] = bf16(y)
 *   fq_rmsnorm_block_quant_ws  codes, row scales and (workspace != NULL) the prepared workspace of the next layer, as fq_rmsnorm_quant_ws
 *
 * Under a norm of its own a row of X with a number that is not finite, or whose squares pass FP32's range, is NaN in H; without one (post_bf16 == NULL) such
 * a number is what the formula makes of it, and the row's others are theirs.  A row whose gate lies outside the gates is NaN in H in either form.  What is
 * NaN or infinite in H does to y, codes and scales what it does in fireq_norm.h.
 *
 *   X_bf16, R_bf16, H_bf16, Y_bf16 [M,K] and gate_bf16 [gates,K] row-major, w_bf16, post_bf16 [K], all 16-byte aligned; gate_rows int32 [M].
 *   eps > 0 and scale finite; K a positive multiple of 8; M < 2^22; 1 <= gates.  H_bf16 may be R_bf16 or X_bf16 itself, Y_bf16 X_bf16 or R_bf16; any
 *   other overlap of an output, or of the workspace, with another array is FQ_ERR_SHAPE.
 * Conventions and status codes are those of fireq.h; M = 0 is a successful no-op.
 */
#ifndef FIREQ_NORM_BLOCK_H
#define FIREQ_NORM_BLOCK_H

#include "fireq.h"

#ifdef __cplusplus
extern "C" {
#endif

int fq_rmsnorm_block(const uint16_t *X_bf16, const uint16_t *post_bf16, const uint16_t *gate_bf16, const int32_t *gate_rows, int gates,
                     float scale, const uint16_t *R_bf16, const uint16_t *w_bf16, float eps, uint16_t *H_bf16, uint16_t *Y_bf16, int M, int K,
                     void *stream);
int fq_rmsnorm_block_quant_ws(const uint16_t *X_bf16, const uint16_t *post_bf16, const uint16_t *gate_bf16, const int32_t *gate_rows,
                              int gates, float scale, const uint16_t *R_bf16, const uint16_t *w_bf16, float eps, uint16_t *H_bf16,
                              uint8_t *A_fp8, float *a_scale, int M, int K, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FIREQ_NORM_BLOCK_H */
