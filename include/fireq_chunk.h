/*
 * fireq_chunk.h -- prompts over the paged INT4 key/value cache of fireq_paged.h: positions on several axes, and the attention of any number
 * of new tokens per sequence with masks, a window, capped scores and a bias by distance.
 *
 * fq_kv4_append_axes   fq_kv4_append with a position for each axis: the pair of dimensions j (0 .. 63) turns by
 *                      cos_sin[positions[axis_of_pair[j]][i]][j], positions being [axes][T]; a pair with axis_of_pair[j] = -1 does not turn.
 *                      axis_of_pair is in host memory and read during the call; 1 <= axes <= 127.  A position outside the table on an axis
 *                      that a pair turns by gives NaN to the row, as there.
 * fq_kv4_attention_chunk_ws   rows starts[b] .. starts[b + 1] - 1 of Q_fp8 [T][Hq][128] are the new tokens of sequence b, the last of its
 *                      seq_lens[b] cached tokens (appended before the call): row i has the place pos = seq_lens[b] - (starts[b + 1] - starts[b]) +
 *                      (i - starts[b]).  It attends to the tokens
 *                          first[i] <= t < end[i],  t > pos - window,  0 <= t < seq_lens[b]
 *                      (first NULL: 0; end NULL: pos + 1, causal; window 0: none), with the scores
 *                          x_t = cap tanh(s_t / cap) - slopes[h] |pos - t|,  s_t = out_scale q . k_t        (cap 0: x = s - ..; slopes NULL: no bias)
 *                      and O[i,h,:] = bf16( sum_t p_t v_t / sum_t p_t ), p_t = exp(x_t).  first and end hold a document's borders, a prefix that is
 *                      seen whole, or any range; a row with no token gets zeros.  A query row in no sequence (before starts[0], behind
 *                      starts[B]) is left as it was.  The products are those of fq_kv4_attention_ws with their error; tanh and the bias are FP32
 *                      (2^-19 of a score), a distance is counted from the row's nearest token on.
 *                      Scores are below 10^7 in magnitude: a row with larger ones may be NaN, and no other is.
 *                      A key or value whose scale is NaN, or a page number outside the cache, gives NaN to the rows that attend to its tokens, and to no
 *                      other.  A sequence longer than max_len or than table_width * page gives NaN to its rows.
 *                      starts int32 [B + 1], not decreasing, 0 .. T (what lies outside is taken as the nearest of these, and rows of
 *                      sequences that overlap are unspecified); first, end int32 [T]; slopes FP32 [Hq], finite (a negative one times any distance, too).
 *                      max_new and max_len are upper bounds of a sequence's rows and of seq_lens that the caller knows; both decide how the work is
 *                      split.  max_new may be wrong: where it is below the truth, that costs time, and scratch for as many parts of T rows as few rows are cut in.
 *                      One max_new chooses the kernel for all sequences: the single tokens of long caches beside a prompt's chunk are better given a call of
 *                      their own (a chunk of 2048 and 40 tokens at up to 29251: 593 us in one call; 205 in two, with the first 41 starts and the last 2, of
 *                      the same Q and O).
 * Scratch: fq_kv4_attention_chunk_workspace_bytes(T, B, Hq, Hkv, max_new, max_len) bytes (often 0), 16-byte aligned, under the rules of
 * fireq_paged.h.
 *
 * window >= 0; cap >= 0 and finite, 0 or at least 2^-60 (one above 2^100 counts as 2^100); out_scale / cap finite; T < 2^23, T * Hq <= 2^25,
 * B <= 65535, T * Hq / 16 + B * Hkv below 2^24, T * (Hq + 2 Hkv) below 2^28 - 16 (append); the other sizes, strides and alignments, outputs that
 * overlap nothing, and status codes as in fireq_paged.h.  T = 0 or B = 0 is a successful no-op.
 */
#ifndef FIREQ_CHUNK_H
#define FIREQ_CHUNK_H

#include "fireq_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

int fq_kv4_append_axes(const uint16_t *QKV_bf16, int64_t ld, const float *cos_sin, int max_positions, const int32_t *positions, int axes,
                       const int8_t *axis_of_pair, const int64_t *slots, int interleaved, uint8_t *Q_fp8, float *q_scale, uint8_t *cache,
                       int64_t page_stride, int64_t head_stride, int pages, int page, int T, int Hq, int Hkv, void *stream);

size_t fq_kv4_attention_chunk_workspace_bytes(int T, int B, int Hq, int Hkv, int max_new, int max_len);
int fq_kv4_attention_chunk_ws(const uint8_t *Q_fp8, const float *q_scale, const uint8_t *cache, int64_t page_stride, int64_t head_stride,
                              int pages, int page, const int32_t *block_table, int table_width, const int32_t *starts,
                              const int32_t *seq_lens, const int32_t *first, const int32_t *end, int window, float cap, const float *slopes,
                              float out_scale, uint16_t *O_bf16, int T, int B, int Hq, int Hkv, int max_new, int max_len, void *workspace,
                              size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FIREQ_CHUNK_H */
