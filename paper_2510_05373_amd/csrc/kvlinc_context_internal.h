// Internal declarations of the attention calls of kvlinc_context.h (not part of the C ABI).
#pragma once

#include "kvlinc_context.h"
#include "kvlinc_internal.h"

namespace kvlinc {

// Splits of a context at most: what a launch is planned with and what the joins are made for.
constexpr int kMaxContextSplits = 32;

// One call as the kernels take it.  Places: row (b, h, i) of q and out is place (b H_q + h) T + i.
struct ContextCall {
  kvlinc_cache cache;
  const _Float16* q;
  const _Float16* k_new;
  const _Float16* v_new;
  const int32_t* n_new;
  int T, window, sinks, gq, splits;
  float* corr;  // [places][kPartStride] {C_d, -, -, -, C_n[128] in the rotated basis}, or NULL: no correction
  float* part;  // [places][splits][kPartStride] as the partial results of the decode kernel, rotated basis; splits > 1 only
  _Float16* out;
  // dequantized tokens [B H_kv][cached_rows][128], values in the rotated basis (launch_dense only): sink_rows rows of the first tokens, then
  // those from window_base on
  _Float16* k_rows;
  _Float16* v_rows;
  // what the rounding of a key to binary16 leaves [B H_kv][cached_rows][128] as FP4 numbers, and the scales of each 32 of them (see low_scores)
  uint32_t* k_low;
  uint32_t* k_low_scale;  // [B H_kv][cached_rows] x 4 bytes
  int cached_rows, sink_rows, row_window;  // row_window: the window that window_base takes, 0 where the rows are all cached tokens
};

// First token that the call's first row sees through its window, down to a multiple of 64: where the dequantized rows start.
constexpr int kTileTokens = 64;
__host__ __device__ inline int window_base(int total, int window) {
  const int low = window > 0 && total - window + 1 > 0 ? total - window + 1 : 0;
  return low & ~(kTileTokens - 1);
}

int launch_rows(const ContextCall& a, int waves, hipStream_t stream);  // up to 64 rows of a KV head; waves of a workgroup: 4 or 8
int launch_windowed(const ContextCall& a, hipStream_t stream);
int launch_tiles(const ContextCall& a, hipStream_t stream);
int launch_dense(const ContextCall& a, hipStream_t stream);
int launch_join(const ContextCall& a, hipStream_t stream);
int launch_prompt_correction(const ContextCall& a, hipStream_t stream);
int launch_read(const kvlinc_cache& c, const int32_t* first, int T, void* k_out, void* v_out, int dtype, bool rotated, hipStream_t stream);

int launch_read_rows(const ContextCall& a, hipStream_t stream);  // k_rows .. k_low_scale

}  // namespace kvlinc
