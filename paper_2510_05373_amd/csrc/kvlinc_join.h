// Partial results of the splits of a context and the correction, and the joining of them to an output row (not part of the C ABI).
#pragma once

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

// ---- results that one workgroup writes and another reads inside the launch ----------------------------------------------------------------
// Stores and loads that go past the caches that are not coherent across the chip (sc0, sc1).  The partial results, and the correction's, of a
// (sequence, KV head) lie together: [head][T][splits] resp. [head][T] rows of kPartStride floats.
constexpr int kCoherent = 1 | 16, kPartBytes = 4 * kPartStride;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(float* p, long long bytes) { return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)bytes, 0x00027000); }
__device__ __forceinline__ void store4(__amdgpu_buffer_rsrc_t r, int at, float a, float b, float c, float d) {
  __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)}, r,
                                         at, 0, kCoherent);
}
__device__ __forceinline__ void store2(__amdgpu_buffer_rsrc_t r, int at, float a, float b) {
  __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)}, r, at, 0, kCoherent);
}
__device__ __forceinline__ float4_t load4(__amdgpu_buffer_rsrc_t r, int at) { return __builtin_bit_cast(float4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, kCoherent)); }
__device__ __forceinline__ float2v_t load2(__amdgpu_buffer_rsrc_t r, int at) { return __builtin_bit_cast(float2v_t, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, kCoherent)); }

// One output row from its 128 numerators (16 lanes, 8 neighbouring channels each): normalised, rotated back.
__device__ __forceinline__ void finish_row(float (&a)[8], float l, int lane, half_t* out) {
  lane8_butterflies(a);
  row16_butterflies<8>(a, lane);
  const float inv = l != 0.0f ? kInvSqrtD / l : 0.0f;  // (0: no tokens)
  u32x4_t h;
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = as_u32(pack_h2(a[2 * i] * inv, a[2 * i + 1] * inv));
  *reinterpret_cast<u32x4_t*>(out + 8 * (lane & 15)) = h;
}
// The correction {C_d, -, -, -, C_n[128]} added (Eq. 5).
__device__ __forceinline__ void add_correction(float (&a)[8], float& l, float m, float c_d, float4_t c0, float4_t c1) {
  const Shares f = shares_of(m, c_d);
  l = fmaf(f.correction, c_d, l * f.softmax);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = fmaf(f.correction, c0[i], a[i] * f.softmax);
    a[4 + i] = fmaf(f.correction, c1[i], a[4 + i] * f.softmax);
  }
}
// The splits of one row joined by 16 lanes: weights by lane, two splits each, and the numerators, kSplitsAhead splits under way at a time, the
// first of them requested together with the maxima.  (A trip to memory, past the caches, is about 2 us of a launch; 16 splits at a time spilled, and
// drafts took 15 % longer.)
constexpr int kSplitsAhead = 8;
__device__ __forceinline__ void join_row(__amdgpu_buffer_rsrc_t part, int at, int splits, float* weights /* LDS, kMaxContextSplits */, int lane, float (&o)[8], float& L, float& M) {
  static_assert(kMaxContextSplits == 32, "a row's 16 lanes take two splits each");
  const int j = lane & 15;
  float4_t u[kSplitsAhead][2];
  auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < kSplitsAhead; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) u[s][k] = load4(part, at + min(s0 + s, splits - 1) * kPartBytes + 16 + 32 * j + 16 * k);
  };
  float2v_t ml[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) ml[k] = load2(part, at + min(j + 16 * k, splits - 1) * kPartBytes);
  request(0);
  const float m[2] = {j < splits ? ml[0][0] : -INFINITY, j + 16 < splits ? ml[1][0] : -INFINITY};
  M = fmaxf(m[0], m[1]);
  M = fmaxf(M, dpp_f<kRowRor1>(M));
  M = fmaxf(M, dpp_f<kRowRor2>(M));
  M = fmaxf(M, dpp_f<kRowRor4>(M));
  M = fmaxf(M, dpp_f<kRowRor8>(M));
  L = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const float w = m[k] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[k] - M);
    weights[j + 16 * k] = w;
    L = fmaf(w, ml[k][1], L);
  }
  L += dpp_f<kRowRor1>(L);
  L += dpp_f<kRowRor2>(L);
  L += dpp_f<kRowRor4>(L);
  L += dpp_f<kRowRor8>(L);
  __builtin_amdgcn_wave_barrier();  // (the 16 lanes are of one wave)
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = 0.0f;
#pragma unroll 1
  for (int s0 = 0;;) {
#pragma unroll
    for (int s = 0; s < kSplitsAhead; ++s) {
      const float w = weights[s0 + s];  // (0 beyond the last)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i] = fmaf(w, u[s][0][i], o[i]);
        o[4 + i] = fmaf(w, u[s][1][i], o[4 + i]);
      }
    }
    s0 += kSplitsAhead;
    if (s0 >= splits) break;
    request(s0);
  }
  __builtin_amdgcn_wave_barrier();
}

}  // namespace
}  // namespace kvlinc
