/*
 * kvlinc_context.h -- attention of prompt rows, attention with a sliding window, and read-back, over the packed cache of kvlinc.h.
 *
 * The conventions of kvlinc.h hold: device pointers of the caller, 16-byte aligned (counts: 4-byte), no allocation, no
 * synchronisation, 0 = enqueued, a negative code = rejected before any launch (KVLINC_EHIP: the runtime refused one).  The calls
 * read the cache and leave all of it as it is, but for split_done, which an attention call may count in and leaves at zero (two
 * calls on the same cache must not overlap in time), and for KVLINC_ST_BOUND in *status.
 *
 * Token t of a sequence that holds n = n_quant + n_res tokens: its key K_t is the dequantized code (t < n_quant) or the window's
 * fp16 row, its value V_t likewise, times H^T (the cache keeps rotated values; with KVLINC_FLAG_SLIDING_VALUES the newest 128
 * tokens have the window's fp16 values).
 *
 * Sliding window and first tokens that stay visible ("sinks"): a query at position p sees token t if
 *     t <= p  and  ( window == 0  or  p - t < window  or  t < sinks ).
 * window = 0 is no limit (sinks is then of no effect); window = 1 leaves the query its own token and the sinks.
 */
#ifndef KVLINC_CONTEXT_H
#define KVLINC_CONTEXT_H

#include "kvlinc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of what kvlinc_cache_read writes. */
enum {
  KVLINC_F16 = 0,
  KVLINC_BF16 = 1,
  KVLINC_F32 = 2
};

/* Bit of *status, beside those of kvlinc.h. */
enum {
  KVLINC_ST_BOUND = 16 /* kvlinc_prompt_attention: a sequence held more tokens than max_context said; its output rows are zeros.
                             kvlinc_attention_mass: likewise; its rows have added nothing */
};

/* Bytes of device scratch kvlinc_prompt_attention needs for T rows a sequence when no sequence holds more than max_context
 * tokens before the call (<= 0: the cache's full capacity).  0 on invalid arguments. */
size_t kvlinc_prompt_workspace_bytes(const kvlinc_cache* cache, int32_t T, int32_t window, int32_t sinks, int32_t max_context);

/*
 * Attention of new tokens ahead of their append ("quantize after attention", Sec. 3.3): a prompt, a chunk of one, or a few
 * drafted tokens.  Row i of sequence b is the token at position n + i; it sees the cached tokens and the new rows up to its own.
 *
 *   q              [B, H_q, T, 128] fp16
 *   k_new, v_new   [B, H_kv, T, 128] fp16, raw rows as kvlinc_append_quantize takes them
 *   n_new          [B] int32 on the device: sequence b has its first n_new[b] (0..T) rows; NULL = T for all.  (A value below 0 is
 *                  read as 0, one above T as T.)  Rows from n_new[b] on are not read, and not written in `out`.
 *   T              rows per (sequence, head), 1 .. 2^24; T and the cache's capacity together below 2^31 - 256 tokens, B * H_kv *
 *                  ceil(T * H_q / H_kv / 16) below 2^24
 *   window, sinks  >= 0, see above
 *   out            [B, H_q, T, 128] fp16, in the original value basis; memory of its own (KVLINC_EINVAL if an input's)
 *   workspace      device scratch of at least kvlinc_prompt_workspace_bytes(cache, T, window, sinks, max_context) bytes, 16-byte
 *                  aligned, contents undefined before and after; NULL where that is 0
 *   max_context    host-side upper bound on the tokens a sequence holds before the call (<= 0: capacity).  It sizes the launch and,
 *                  for more than 512 rows a KV head (T * H_q / H_kv), the room for dequantized tokens (580 bytes each): a
 *                  sequence that holds more than there is room for gets zeros in its rows, and KVLINC_ST_BOUND is set.
 *                  Where nothing is cached yet, 1 says so: without it a first prompt of that many rows reserves the room of a
 *                  full cache (16 sequences of up to 131072 tokens, 8 KV heads: 9.7 GB) and looks through it.
 *
 * out[b, h, i] = ( sum_t w_t V_t + phi_q(q) S H^T ) / ( sum_t w_t + phi_q(q) P ),  w_t = exp(q K_t / sqrt 128)
 * over the tokens that row i sees; the phi terms (Eq. 5) with the adapters only.  The states S, P stand for all quantized tokens:
 * with adapters, window > 0 is refused, and so is KVLINC_FLAG_ALG1_LITERAL.  Where nothing is quantized yet (S = P = 0) it is the
 * softmax alone, however low the logits.  The cache may end in a partial group.
 *
 * Arithmetic: matrix products of binary16 operands with binary32 sums; softmax weights, and values where they are dequantized
 * ahead of a product, are rounded to binary16 once; running maximum, sums and numerators are binary32.  Keys are exact for up to
 * 64 rows of a KV head; for more they are binary16 numbers, and what that leaves is held to a few percent of 2^-12 of the
 * largest of 32 channels (keys with an offset of 300 in some channels: outputs 1e-3 to 2e-3 of their norm off, without it 3e-4).
 * A key or value among the new rows that is not finite makes the rows that see it not finite (but for a key that is infinite and
 * gets the weight 0), and no others: earlier rows and rows whose window has passed it stay right.  (The append then refuses the sequence.)
 * Results do not depend on the order in which the workgroups run.
 */
int kvlinc_prompt_attention(const kvlinc_cache* cache, const kvlinc_half* q, const kvlinc_half* k_new, const kvlinc_half* v_new,
                            const int32_t* n_new, int32_t T, int32_t window, int32_t sinks, kvlinc_half* out, void* workspace,
                            size_t workspace_bytes, int32_t max_context, void* stream);

/* Bytes of device scratch kvlinc_decode_attention_windowed needs; max_context as below.  0 on invalid arguments. */
size_t kvlinc_decode_windowed_workspace_bytes(const kvlinc_cache* cache, int32_t window, int32_t sinks, int32_t max_context);

/*
 * One decode step of a layer with a sliding window: kvlinc_decode_attention (the query's own token, at position n - 1, is already
 * appended) over the tokens that the window and the sinks leave visible.  Only their groups are read.
 *
 *   q, out         [B, H_q, 128] fp16; out may be q (other overlaps: KVLINC_EINVAL)
 *   window, sinks  >= 0, see above; window = 0: all tokens
 *   workspace      at least kvlinc_decode_windowed_workspace_bytes(cache, window, sinks, max_context) bytes, 16-byte aligned
 *   max_context    host-side upper bound on n_quant + n_res (<= 0: capacity); it only sizes the launch
 *
 * Needs a cache without adapters: the correction's states stand for all quantized tokens.  A sequence with no tokens yields zeros.
 */
int kvlinc_decode_attention_windowed(const kvlinc_cache* cache, const kvlinc_half* q, int32_t window, int32_t sinks, kvlinc_half* out,
                                     void* workspace, size_t workspace_bytes, int32_t max_context, void* stream);

/*
 * Keys and values of T tokens of every sequence as a plain attention would take them.
 *
 *   first          [B] int32 on the device: row i is token first[b] + i; NULL = 0 for all.  (A value below 0 is read as 0.)
 *   T              rows, 1 .. 2^30; B * H_kv * T at most 2^40
 *   k_out, v_out   [B, H_kv, T, 128] of type dtype (KVLINC_F16, KVLINC_BF16, KVLINC_F32); either may be NULL.  Rows of tokens
 *                  that the sequence does not hold are left as they are.  The two do not overlap.
 *   rotated        0: values in the original basis, V_t;  1: in the rotated basis they are stored in.
 *
 * A number is dequantized and rotated in binary32 and rounded to dtype once; one beyond the largest finite binary16 number (the
 * quantizer's own rounding can put it there) is stored as +-65504 in KVLINC_F16.
 */
int kvlinc_cache_read(const kvlinc_cache* cache, const int32_t* first, int32_t T, void* k_out, void* v_out, int32_t dtype,
                      int32_t rotated, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KVLINC_CONTEXT_H */
