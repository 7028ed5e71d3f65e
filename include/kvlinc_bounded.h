/*
 * kvlinc_bounded.h -- long generation in a cache of bounded size: positions of new rows, accumulated attention weight, eviction by it.
 *
 * The conventions of kvlinc.h hold: device pointers of the caller, 16-byte aligned (32-bit numbers: 4-byte), no allocation, no synchronisation, 0 =
 * enqueued, a negative code = rejected before any launch (KVLINC_EHIP: the runtime refused one).  Two calls on the same cache must not overlap
 * in time.
 *
 * The mass of a group.  The tokens of a (sequence, KV head) lie in groups of 128; a sequence of n_quant and n_res tokens has the groups
 * 0 .. c - 1, c = ceil(n_quant / 128), and the tokens of its fp16 window, which a later append makes group c.  mass [B, H_kv, max_groups + 1], binary32,
 * holds for each of these the attention weight that its tokens have received; slot c is the window's, so that a group keeps what its tokens received
 * before they were quantized.  A call adds, for every query row that it is given,
 *     w_t = exp(q K_t / sqrt 128) / sum_u exp(q K_u / sqrt 128)          (u: the tokens that the row sees)
 * to the slot of token t, summed over the query heads of the KV head: each row that sees a token adds 1 to a KV head's slots for each of its heads.
 * Slots beyond c are not touched by the calls that add; new groups start from what is there: zero them once, kvlinc_cache_evict keeps them zero.
 *
 * None of the calls that take weights or evict works with the adapters of the correction (KVLINC_EINVAL): its states stand for all tokens
 * ever quantized.  They take caches with B * H_kv below 2^24, B * H_kv * (max_groups + 1) below 2^26 and room for less than 2^31 - 256 tokens a sequence.
 */
#ifndef KVLINC_BOUNDED_H
#define KVLINC_BOUNDED_H

#include "kvlinc_context.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- positions ---- */

/* Rotary positions.  Pair i (0 <= i < channels / 2) of a row at position p is turned by the angle p freq[i]:
 *     (x, y) -> magnitude (x cos - y sin, x sin + y cos).
 * Channels from `channels` on pass as they are. */
typedef struct kvlinc_rotation {
  int32_t channels;    /* rotated channels: even, 2..128, the first ones of a head */
  int32_t interleaved; /* 0: pair i is channels i and i + channels / 2;  1: channels 2 i and 2 i + 1 */
  float magnitude;     /* finite; 1 unless the scaling for long contexts has one */
  const double* freq;  /* [channels / 2] radians per position, on the device, 16-byte aligned */
} kvlinc_rotation;

/* Rows of one tensor: sequence b, head h, token i has its 128 numbers, contiguous, at in + b sequence_stride + h head_stride + i token_stride
 * (strides in numbers, 0 or more, multiples of 16 bytes).  out is [B, heads, T, 128], contiguous: as kvlinc_append_quantize and kvlinc_prompt_attention
 * take it (at T = 1, as kvlinc_decode_attention does).  out may be in itself where that is contiguous and of the same type; otherwise it shares no
 * memory with what lies between the first and the last row of an input. */
typedef struct kvlinc_rows {
  const void* in;
  void* out;
  int64_t sequence_stride, head_stride, token_stride;
} kvlinc_rows;

/*
 * Queries and keys of T new tokens of every sequence rotated to their positions, values taken along as they are, to the layout and type of the
 * cache's calls: what stands between a layer's projections and kvlinc_append_quantize, kvlinc_prompt_attention or a decode step.
 *
 *   cache      B, H_q, H_kv and, where counted is 1, the counters n_quant and n_res
 *   q, k, v    rows of H_q, H_kv, H_kv heads; each may be NULL, not all three
 *   T          rows per sequence, 1 .. 2^24; B * T at most 2^26 - 4
 *   n_new      [B] int32 on the device: sequence b has its first n_new[b] (0..T) rows; NULL = T for all.  (A value below 0 is read as 0, one
 *              above T as T.)  Rows from n_new[b] on are not read, and not written.
 *   first      [B] int32 on the device, NULL = 0 for all
 *   depth      [B, T] int32 on the device, NULL: 0, 1, 2, ... (drafted trees have rows of the same depth)
 *   counted    1: the position of row i is n_quant[b] + n_res[b] + first[b] + depth[b][i], ahead of the append (first: the tokens that are not in
 *              the cache any more, see kvlinc_cache_evict);  0: first[b] + depth[b][i]
 *   dtype_in, dtype_out   KVLINC_F16, KVLINC_BF16 or KVLINC_F32, of all three tensors
 *
 * Angles are formed and reduced in binary64 (exact to 2^-51 of p freq), sines, cosines and products in binary32; a number is rounded to dtype_out
 * once.  (A finite number beyond the range of dtype_out becomes infinite, which the append reports.)
 */
int kvlinc_rotary(const kvlinc_cache* cache, const kvlinc_rotation* rotation, const kvlinc_rows* q, const kvlinc_rows* k, const kvlinc_rows* v,
                  int32_t T, const int32_t* n_new, const int32_t* first, const int32_t* depth, int32_t counted, int32_t dtype_in,
                  int32_t dtype_out, void* stream);

/* ---- accumulated attention weight ---- */

/* Bytes of device scratch kvlinc_decode_attention_mass needs; max_context as there.  0 on invalid arguments. */
size_t kvlinc_decode_mass_workspace_bytes(const kvlinc_cache* cache, int32_t max_context);

/*
 * One decode step over the whole cache (as kvlinc_decode_attention: the query's own token is already appended) that also accumulates the mass:
 *     mass_out[b, g, j] = decay mass[b, g, j] + weights of the query's heads on the tokens of slot j,      j = 0 .. c.
 *
 *   q, out         [B, H_q, 128] fp16; out may be q (other overlaps: KVLINC_EINVAL)
 *   mass           [B, H_kv, max_groups + 1] binary32, or NULL: zeros
 *   decay          0 .. 1; with 0, mass is not read
 *   mass_out       [B, H_kv, max_groups + 1] binary32; may be mass (other overlaps: KVLINC_EINVAL).  Slots beyond c are left as they are.
 *   workspace      at least kvlinc_decode_mass_workspace_bytes(cache, max_context) bytes, 16-byte aligned, contents undefined before and after
 *   max_context    host-side upper bound on n_quant + n_res (<= 0: capacity); it only sizes the launch, results do not depend on it but for the
 *                  order of sums
 *
 * A sequence with no tokens yields zeros and decay mass.  Scores are those of exact products with the dequantized keys to 2^-16 of each;
 * sums are binary32, and do not depend on the order in which the workgroups run.
 */
int kvlinc_decode_attention_mass(const kvlinc_cache* cache, const kvlinc_half* q, kvlinc_half* out, const float* mass, float decay, float* mass_out,
                                 void* workspace, size_t workspace_bytes, int32_t max_context, void* stream);

/* Bytes of device scratch kvlinc_attention_mass needs for T rows a sequence when no sequence holds more than max_context tokens (<= 0: the cache's
 * full capacity).  0 on invalid arguments. */
size_t kvlinc_attention_mass_workspace_bytes(const kvlinc_cache* cache, int32_t T, int32_t max_context);

/*
 * The mass that T query rows of every sequence add, without their output rows (no values are read): the last rows of a prompt, say, after it has
 * been appended.  Row i of the r rows of sequence b is the query of its token n - r + i, n = n_quant + n_res: the rows' own tokens are the newest in the
 * cache.  It sees the tokens up to its own; a row ahead of the first token (r > n) sees nothing and adds nothing.
 *     mass_out[b, g, j] = decay mass[b, g, j] + weights of the rows' heads on the tokens of slot j,      j = 0 .. c.
 *
 *   q              [B, H_q, T, 128] fp16
 *   n_rows         [B] int32 on the device: sequence b has its first n_rows[b] (0..T) rows; NULL = T for all.  (A value below 0 is read as 0, one
 *                  above T as T.)  Rows from n_rows[b] on are not read.
 *   T              rows per (sequence, head), 1 .. 2^20; B * H_kv * ceil(T * H_q / H_kv / 64) below 2^22
 *   mass, decay, mass_out   as above
 *   workspace      at least kvlinc_attention_mass_workspace_bytes(cache, T, max_context) bytes, 16-byte aligned: 4 bytes for every row of a query head
 *                  and group that max_context tokens can have (all rows of a prompt of 32768 tokens, 32 query heads: 1.1 GB, of 131072: 17.2 GB;
 *                  a prompt that is appended in chunks, with a call behind each of them, needs that of a chunk)
 *   max_context    host-side upper bound on n_quant + n_res (<= 0: capacity).  It sizes the workspace: the rows of a sequence that holds more tokens
 *                  (max_context + 1 or more) add nothing, and KVLINC_ST_BOUND is set in *status.
 */
int kvlinc_attention_mass(const kvlinc_cache* cache, const kvlinc_half* q, const int32_t* n_rows, int32_t T, const float* mass, float decay,
                          float* mass_out, void* workspace, size_t workspace_bytes, int32_t max_context, void* stream);

/* ---- eviction ---- */

/* Bytes of device scratch kvlinc_cache_evict needs.  0 on invalid arguments. */
size_t kvlinc_cache_evict_workspace_bytes(const kvlinc_cache* cache);

/*
 * Every sequence that holds more than `limit` groups is cut to `keep` of them: of each KV head, the first `first`, the newest `last` and those
 * with the largest mass between them (of equal ones, the older; one that is not a number counts as less than any other).  Groups are kept or dropped
 * whole: the keys of a group share their scales.  What is kept stays in its order and bit for bit, codes, scales and window; n_quant becomes smaller by
 * 128 tokens for every dropped group.  The tokens in the window all stay.
 *
 *   from           the cache
 *   to             where the kept groups, the window and the counters go: from itself (in place; the same descriptor in all of its buffers), or a cache
 *                  of the same B, H_q, H_kv, R, bits and flags that shares no memory with it, and has room for `limit` groups, or as many
 *                  as from has room for.  Storage of it beyond its counters may be overwritten; status stays as it is, split_done, which may be counted in, zero.
 *   mass           [B, H_kv, from->max_groups + 1] binary32
 *   mass_out       [B, H_kv, to->max_groups + 1] binary32: the mass of what is kept, the window's behind it, and zeros to the end.  May be mass
 *                  where both have room for as many groups.
 *   keep, limit    1 <= keep <= limit
 *   first, last    first >= 0, last >= 1 (the newest group always stays: a later append, and KVLINC_FLAG_SLIDING_VALUES, build on it),
 *                  first + last <= keep
 *   offset         [B] int32 or NULL (zeros): tokens of the sequence that earlier calls have dropped
 *   offset_out     [B] int32 or NULL: offset and those that this call drops, what the `first` of kvlinc_rotary takes.  May be offset.
 *   kept           [B, H_kv, to->max_groups] int32 or NULL: the slot in `from` that each kept group had; entries beyond them are left as they are
 *   workspace      at least kvlinc_cache_evict_workspace_bytes(from) bytes, 16-byte aligned
 */
int kvlinc_cache_evict(const kvlinc_cache* from, const kvlinc_cache* to, const float* mass, float* mass_out, int32_t keep, int32_t limit,
                       int32_t first, int32_t last, const int32_t* offset, int32_t* offset_out, int32_t* kept, void* workspace,
                       size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KVLINC_BOUNDED_H */
