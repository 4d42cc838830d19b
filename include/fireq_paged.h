/*
 * fireq_paged.h -- decode attention on a paged INT4 key/value cache: the position rotation and quantisation that fill it,
 * the attention of one new token per sequence over it, alone or behind a prefix that all sequences share, and its read-back.
 *
 * Queries are FP8 with a scale per token and head, keys and values INT4 with an E4M3 scale per token and head (Sec. 3.2.1;
 * Sec. 2.1: "INT4 with FP8 scaling factors"); heads are 128 wide.  Query head h attends to key/value head h / (Hq / Hkv).
 *
 * The cache is uint8 [pages][Hkv][page / 16][2080], page a positive multiple of 16: 2080 bytes ("tile") hold 16 tokens of a
 * head.  A code is the INT4 number + 8 (0..15).
 *   keys    byte 256 g + 16 t + j        token t, dimension 32 g + j (low nibble) and 32 g + 16 + j (high)
 *   values  byte 1024 + 256 p + 16 n + 4 m + b
 *                                        token 4 p + (0, 2, 1, 3)[b], channel n + 32 m (low) and n + 32 m + 16 (high)
 *   scales  byte 2048 + 8 p + i          E4M3 scale of the key of token 4 p + i; + 4: of its value
 * page_stride (below 2^36) and head_stride are in bytes, positive multiples of 16 (a page of a head is contiguous; head_stride is at least
 * page / 16 * 2080 and pages do not overlap).  Slot s is token s % page of page s / page.  A fresh cache may hold anything: no
 * call reads a token that was not appended, or lets its bytes count.
 *
 * fq_kv4_append   T rows of QKV_bf16 [T][ld]: Hq query, Hkv key and Hkv value heads of 128 (ld >= 128 (Hq + 2 Hkv), a
 *                 multiple of 8).  With (c, s) = cos_sin[positions[i]][j], FP32 [max_positions][64][2], the pair (a, b) of
 *                 dimensions (j, j + 64), or (2 j, 2 j + 1) where interleaved != 0, of every query and key head becomes
 *                     (a c - b s, b c + a s),
 *                 products and sum in FP64, rounded once to FP32.  Then
 *                     queries         q_scale = max |q| / 448 (1 for zeros), Q_fp8 = E4M3 nearest-even of q / q_scale
 *                     keys, values    sigma = E4M3 nearest-even of min(max |x| / 7, 448), code = clamp(round_half_even(x / sigma),
 *                                     -8, 7), 0 where sigma is 0; FP32 quotients
 *                 (sigma's least steps are 2^-9 and there is no further factor: a key or value head of max |x| <= 7 * 2^-10,
 *                 0.0068, is kept as zeros, and one below 0.012 in few steps.  Layers with heads that small scale their key projection by
 *                 a power of two and out_scale back, their value projection and the output layer's w_tscale back)
 *                 and key and value go to slot slots[i].  A negative slot is padding: nothing is cached.  Two rows with one slot
 *                 leave either's bytes.  What cannot be done shows: a head with a number that is not finite gets the scale NaN
 *                 (codes 0); a position outside the table, or a slot behind the cache's end (nothing is cached), gives
 *                 NaN q_scales to the whole row and, where there is a slot, NaN scales in it.
 *                 Q_fp8 [T][Hq][128], q_scale [T][Hq].
 * fq_kv4_read     K_bf16, V_bf16 [n][Hkv][128] = sigma * code (exact in bf16) of the tokens in `slots`; zeros for a negative
 *                 slot, NaN for one behind the cache's end.
 * fq_kv4_attention_ws   O[b,h,:] = bf16( sum_t p_t v_t / sum_t p_t ), p_t = exp(out_scale q . k_t), over the tokens
 *                 t < seq_lens[b], token t in page block_table[b][t / page] (row b at block_table + b * table_width).  A
 *                 sequence with no token (a length <= 0) gets zeros.  Scores are sums q_scale sigma out_scale
 *                 (sum_d q_d (code_d + 8) - 8 sum_d q_d) on the FP8 matrix cores, whose products are exact and are aligned to the
 *                 largest of an instruction before they are added: a score lies within 2^-12 of the largest
 *                 |q_scale q_d sigma out_scale| max(code_d + 8, 8) of its token (measured: 2^-13), and within FP32's
 *                 roundings of its factors, of the exact one.  A query with one channel far above the others feels it in the
 *                 others.  Probabilities, relative to a running maximum, enter the FP32 sums as fp16 numbers; sigma * code is exact.
 *                 out_scale > 0; max_len is an upper bound of seq_lens that the caller knows.  It decides how the work is
 *                 split, and parts that no sequence has are dispatched and joined all the same: 64 sequences of 1000 tokens
 *                 (32 / 8 heads) take 16 us with max_len 1000, 24 with 32768, 54 with 131072; 32 of them 9.9, 13.7 and 13.7.
 *                 A sequence longer than it, or than table_width * page, or a page number outside the cache within a sequence's
 *                 length, gives NaN for that sequence.
 * fq_kv4_attention_prefix_ws   the same where every sequence attends to prefix_len tokens in prefix_pages first, and then
 *                 to its own seq_lens[b] tokens: the prefix is read and unpacked for up to 32 query rows at a time, not for
 *                 every sequence (unless that is less work than sharing it).
 * Scratch: fq_kv4_attention_workspace_bytes(B, Hq, Hkv, max_len, prefix_len) bytes, 16-byte aligned (prefix_len 0: without
 * prefix; 0 bytes for sizes that the calls refuse); it may be
 * reused or freed once the work enqueued by the call has finished, and calls that overlap in time need scratch of their own.
 *
 * Outputs (Q_fp8, q_scale, the cache of an append, K, V, O) and scratch overlap neither each other nor anything that the call reads
 * (FQ_ERR_SHAPE).  A cache is its tiles: what lies between them, other layers of one pool say, may be an output.
 *
 * Q_fp8, cache, QKV_bf16, cos_sin, K, V, O: 16-byte aligned.  Conventions and status codes are those of fireq.h; T, n or B = 0
 * is a successful no-op.  Hq is a multiple of Hkv; B, Hq <= 65535, B * Hq <= 2^23, max_len and prefix_len <= 2^30, T < 2^23, T * (Hq + 2 Hkv) and n * Hkv below 2^28 - 16, fewer than 2^32 tiles a head.
 */
#ifndef FIREQ_PAGED_H
#define FIREQ_PAGED_H

#include "fireq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FQ_KV4_TILE_TOKENS 16
#define FQ_KV4_TILE_BYTES 2080

int fq_kv4_append(const uint16_t *QKV_bf16, int64_t ld, const float *cos_sin, int max_positions, const int32_t *positions,
                  const int64_t *slots, int interleaved, uint8_t *Q_fp8, float *q_scale, uint8_t *cache, int64_t page_stride,
                  int64_t head_stride, int pages, int page, int T, int Hq, int Hkv, void *stream);
int fq_kv4_read(const uint8_t *cache, int64_t page_stride, int64_t head_stride, int pages, int page, const int64_t *slots,
                uint16_t *K_bf16, uint16_t *V_bf16, int n, int Hkv, void *stream);

size_t fq_kv4_attention_workspace_bytes(int B, int Hq, int Hkv, int max_len, int prefix_len);
int fq_kv4_attention_ws(const uint8_t *Q_fp8, const float *q_scale, const uint8_t *cache, int64_t page_stride, int64_t head_stride,
                        int pages, int page, const int32_t *block_table, int table_width, const int32_t *seq_lens, float out_scale,
                        uint16_t *O_bf16, int B, int Hq, int Hkv, int max_len, void *workspace, size_t workspace_bytes, void *stream);
int fq_kv4_attention_prefix_ws(const uint8_t *Q_fp8, const float *q_scale, const uint8_t *cache, int64_t page_stride,
                               int64_t head_stride, int pages, int page, const int32_t *prefix_pages, int prefix_len,
                               const int32_t *block_table, int table_width, const int32_t *seq_lens, float out_scale,
                               uint16_t *O_bf16, int B, int Hq, int Hkv, int max_len, void *workspace, size_t workspace_bytes,
                               void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FIREQ_PAGED_H */
