/*
 * fireq_norm.h -- root-mean-square norm in front of a quantised layer, with the residual stream's addition.
 *
 *   H[m,k] = bf16( X[m,k] + R[m,k] )                     (R == NULL: H is X itself and is not written)
 *   y[m,k] = H[m,k] * w[k] / sqrt( (1/K) sum_k H[m,k]^2 + eps )
 *
 * The sum of squares and y are FP32; y is not rounded to bf16 on its way to the codes.
 *
 *   fq_rmsnorm           Y_bf16[m,k] = bf16(y)           (the norm behind the last block)
 *   fq_rmsnorm_quant_ws  a_scale[m] = max_k |y| / 448 (1 for a row of zeros), A_fp8[m,k] = E4M3 nearest-even of y / a_scale:
 *                        the operands of fq_w4a8_gemm_ws.  With workspace != NULL (fq_w4a8_gemm_workspace_bytes(M,N,K) bytes
 *                        or more; K a multiple of 128, at most 16384 then) the call also prepares that workspace
 *                        (workspace_prepared = 1 there), as fq_quantize_act_ws does; where that size is 0 (M <= 64) it may
 *                        be NULL.
 *
 * A row with a number that is not finite, or whose squares, sum, products with w or y pass FP32's range, gets the scale NaN and
 * codes of zero: every output of the layer behind it is NaN in that row, and no code is.  (fq_rmsnorm: NaN throughout, and
 * infinity for a single y past the range.)
 *
 *   X_bf16, R_bf16, H_bf16, Y_bf16 [M,K] row-major, 16-byte aligned; w_bf16 [K], 16-byte aligned; eps > 0, finite.
 *   K a positive multiple of 8; M < 2^22.  H_bf16 is written where R_bf16 is given (both or none, FQ_ERR_NULL) and may be R_bf16 or
 *   X_bf16 itself; any other overlap of H or Y with an input is FQ_ERR_SHAPE (Y_bf16 may be X_bf16 or R_bf16), and so
 *   is any of a_scale or of the workspace with another array of the call.
 * Conventions and status codes are those of fireq.h; M = 0 is a successful no-op.
 */
#ifndef FIREQ_NORM_H
#define FIREQ_NORM_H

#include "fireq.h"

#ifdef __cplusplus
extern "C" {
#endif

int fq_rmsnorm(const uint16_t *X_bf16, const uint16_t *R_bf16, const uint16_t *w_bf16, float eps, uint16_t *H_bf16,
               uint16_t *Y_bf16, int M, int K, void *stream);
int fq_rmsnorm_quant_ws(const uint16_t *X_bf16, const uint16_t *R_bf16, const uint16_t *w_bf16, float eps, uint16_t *H_bf16,
                        uint8_t *A_fp8, float *a_scale, int M, int K, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FIREQ_NORM_H */
