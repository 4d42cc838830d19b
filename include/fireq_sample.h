/*
 * fireq_sample.h -- a token for each row of logits, from a given uniform random number.
 *
 * Row b of logits [B][ld] has V logits x, T = temperature[b], k = top_k[b], p = top_p[b], m = min_p[b] and u = u[b] (a NULL array: T = 1, and no
 * filter).  Tokens stand in the order of their logits, the larger first, the lower index first among equals.  Kept are
 *     of all tokens those with (x - max x) / T >= log m    (m <= 0: all; m > 1 counts as 1)
 *     of these the first k                                  (k <= 0: all)
 *     of these the least first number whose mass, sum exp(x / T), is at least p times theirs   (p >= 1: all; p <= 0: the first)
 * token[b] is the first token, by index, at which the kept mass up to it passes u times the whole kept mass (u is taken as one of [0, 1 - 2^-24]), and
 * logprob[b] = log softmax(x / T)[token], over all V.  T = 0 takes the best token, and its log-probability at T = 1.  Any other T counts as
 * one of 2^-100 .. 2^100.
 *
 * -infinity is a token of no mass.  Exponentials are FP32 and sums those of whole numbers, of which the largest of the row, or of a part of it, has
 * 2^32 - 2^8 (the log-probability's may be FP32's): a token below 2^-32 of the row's best may be taken as one of no mass.  Results do not depend on the
 * order in which anything runs.
 * A row with a NaN or +infinity, with no token above -infinity, with T negative or not finite, or with u, p or m NaN, gives token -1 and
 * logprob NaN.
 *
 * fq_sample_bf16_ws, fq_sample_fp32_ws   logits in bf16, in FP32; aligned to their size, ld >= V; logprob may be NULL.
 * Scratch: fq_sample_workspace_bytes(B, V) bytes (0 up to V = 32761), 16-byte aligned; it may be reused or freed once the work enqueued by the call
 * has finished, and calls that overlap in time need scratch of their own.
 * 1 <= V <= 2^20, B <= 65535; outputs and scratch overlap neither each other nor an input (FQ_ERR_SHAPE).  Conventions and status codes are those of
 * fireq.h; B = 0 is a successful no-op.
 */
#ifndef FIREQ_SAMPLE_H
#define FIREQ_SAMPLE_H

#include "fireq.h"

#ifdef __cplusplus
extern "C" {
#endif

size_t fq_sample_workspace_bytes(int B, int V);
int fq_sample_bf16_ws(const uint16_t *logits, int64_t ld, const float *u, const float *temperature, const int32_t *top_k,
                      const float *top_p, const float *min_p, int32_t *token, float *logprob, int B, int V, void *workspace,
                      size_t workspace_bytes, void *stream);
int fq_sample_fp32_ws(const float *logits, int64_t ld, const float *u, const float *temperature, const int32_t *top_k, const float *top_p,
                      const float *min_p, int32_t *token, float *logprob, int B, int V, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FIREQ_SAMPLE_H */
