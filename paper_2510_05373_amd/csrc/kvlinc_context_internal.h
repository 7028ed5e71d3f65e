// Internal declarations of the attention calls of kvlinc_context.h (not part of the C ABI).
#pragma once

#include "kvlinc_context.h"
#include "kvlinc_internal.h"

namespace kvlinc {

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
};

int launch_rows(const ContextCall& a, bool prompt, hipStream_t stream);
int launch_tiles(const ContextCall& a, hipStream_t stream);
int launch_join(const ContextCall& a, bool prompt, hipStream_t stream);
int launch_prompt_correction(const ContextCall& a, hipStream_t stream);
int launch_read(const kvlinc_cache& c, const int32_t* first, int T, void* k_out, void* v_out, int dtype, bool rotated, hipStream_t stream);

}  // namespace kvlinc
