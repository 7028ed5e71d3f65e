// Internal declarations of the calls of kvlinc_bounded.h (not part of the C ABI).
#pragma once

#include "kvlinc_bounded.h"
#include "kvlinc_internal.h"

namespace kvlinc {

// ---- positions ----
struct RotaryRows {
  const void* in;
  void* out;
  long long sequence_stride, head_stride, token_stride;
  int heads;  // 0: no such rows
};
struct RotaryCall {
  RotaryRows rows[3];  // queries, keys, values
  const double* freq;
  const int32_t* n_quant;  // NULL: positions are not counted from the cache
  const int32_t* n_res;
  const int32_t* first;
  const int32_t* depth;
  const int32_t* n_new;
  float magnitude;
  int channels, B, T, heads, steps;  // heads: of all three; steps: of 8 heads that a wave takes
};
int launch_rotary(const RotaryCall& a, bool interleaved, int dtype_in, int dtype_out, hipStream_t stream);

// ---- accumulated attention weight ----
// One call as the kernels take it.  Slots of a (sequence, KV head): a group each, and the window's behind the last.
struct MassCall {
  kvlinc_cache cache;
  const _Float16* q;
  const int32_t* n_rows;
  const float* mass;  // NULL: zeros
  float* mass_out;
  float decay;
  int T, gq;
  int units;          // decode: workgroups of a KV head, B or more
  _Float16* out;
  float* part;        // decode: partial results of the splits as in kvlinc_context_internal.h; splits > 1 only
  unsigned long long* sums;  // decode: [B H_kv][slots][8] pairs {reference, sum of weights} of a head, see kvlinc_decode_mass.hip
  float* lse;         // rows: [B H_kv][slots][rows] log2 of a row's sum of weights over the slot's tokens
  float* row_lse;     // rows: [B H_kv][rows] the same over all tokens it sees
  long long slots;
  int bound;          // rows: a sequence of more tokens is not taken; one of so many needs no more than `slots`
  int rows;           // of a (sequence, KV head), up to a multiple of 16
};
int launch_decode_mass(const MassCall& a, hipStream_t stream);
int launch_attention_mass(const MassCall& a, hipStream_t stream);

// ---- eviction ----
// Caches of few groups, whose keys every workgroup's wave holds (and a sequence's pairs are counted in half a word): 256 pairs of 300 groups at 2 bits, 32 kept,
// 38.2 us for 42.1 with a launch of its own to select, of 500 40.8 for 42.3, of 1000 49.2 for 45.2; 128 pairs at 4 bits, 64 kept of 256 59.7 for 68.9,
// of 500 72.7 for 66.3.
inline bool evicts_in_one_launch(const kvlinc_cache& c) { return c.max_groups <= (c.bits == 2 ? 512 : 256) && c.H_kv < (1 << 15); }
struct EvictCall {
  kvlinc_cache from, to;
  const float* mass;
  float* mass_out;
  int keep, limit, first, last;
  const int32_t* offset;
  int32_t* offset_out;
  int32_t* kept;
  // where a launch of its own selects:
  int32_t* source;  // [B H_kv][stride] slots of the kept groups
  int32_t* count;   // [B H_kv][2] how many, and the first that has another slot than before
  long long stride;
  bool in_place;
  bool counted;     // something is written over what all workgroups of a pair read
};
int launch_evict(const EvictCall& a, hipStream_t stream);

}  // namespace kvlinc
