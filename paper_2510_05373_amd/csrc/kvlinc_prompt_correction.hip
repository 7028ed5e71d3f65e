// The linear correction of prompt rows (Sec. 3.2, Eq. 5-6): C_n = phi_q(q) S and C_d = phi_q(q) P of every row, in the rotated basis.
//
// A workgroup takes 128 tokens of one head, a wave 16, one a column of the products (kvlinc_features.h).
// The eight waves bring the weights and the state to LDS together, half of the features at a time, as operands: read by every wave for itself, 128 KB
// for 32 tokens, they took twice as long (8192 tokens of 32 heads with what reads the results: 200 us, 109 so; 128 tokens 24 and 11; 32 tokens a wave: 122).
// Bound: the results, 528 bytes a row, written and read again (0.28 GB, 53 us of the 109), and the operands from L2.
#include <hip/hip_runtime.h>

#include "kvlinc_context_internal.h"
#include "kvlinc_features.h"

namespace kvlinc {
namespace {

constexpr int kCorrWaves = 8, kCorrTokens = 16 * kCorrWaves;
// Grid: blocks of 128 tokens fastest, then (sequence, query head).
__global__ __launch_bounds__(64 * kCorrWaves, 4) void prompt_correction_kernel(ContextCall a, int blocks) {
  __shared__ u32x4_t sW[2][4][4][64];  // operands of a half of the features, as lanes take them: weights [64-feature block][32 channels][tile]
  __shared__ u32x4_t sS[2][8][2][64];  // and the state [64-feature block][16 channels][8 features of a lane]
  const kvlinc_cache& c = a.cache;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, g = lane >> 4;
  const long long bh = blockIdx.x / blocks;  // b H_q + h
  const int first = (int)(blockIdx.x - bh * blocks) * kCorrTokens, token = first + 16 * wave + j, b = (int)(bh / c.H_q), h = (int)(bh - (long long)b * c.H_q);
  const int T = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T;
  if (first >= T) return;
  const bool idle = first + 16 * wave >= T;  // (the wave only helps to bring the operands)
  const long long kv = (long long)b * c.H_kv + h / a.gq;

  half8_t q[4];  // channels 32 s + 8 g + 0..7
  const u32x4_t* src = reinterpret_cast<const u32x4_t*>(a.q + (bh * a.T + min(token, T - 1)) * kHeadDim) + g;
#pragma unroll
  for (int s = 0; s < 4; ++s) q[s] = as_h8(src[4 * s]);
  float4_t acc[8];
  float den = 0.0f;
#pragma unroll
  for (int n = 0; n < 8; ++n) acc[n] = float4_t{0.f, 0.f, 0.f, 0.f};
  const half_t* S = reinterpret_cast<const half_t*>(c.S16) + kv * (128 * 64 * 4);
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    const half_t* W = reinterpret_cast<const half_t*>(c.Wq) + ((long long)h * 2 + half) * kHeadDim * 128;
    if (half != 0) __syncthreads();
    {  // a wave has one block of features and 32 channels of the weights, and 16 channels of the state
      const int fb = wave >> 2, s = wave & 3, n = wave;
      u32x4_t w[4];
      weight_operands(W, s, fb, j, g, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) sW[fb][s][i][lane] = w[i];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int e = 0; e < 2; ++e) sS[f][n][e][lane] = state_operand(S, 128 * half + 64 * f + 16 * g + 8 * e, 16 * n + j);
    }
    __syncthreads();
    if (idle) continue;
    float4_t x[2][4];  // [64-feature block][tile]
#pragma unroll
    for (int fb = 0; fb < 2; ++fb) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[fb][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[fb][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(sW[fb][s][i][lane]), q[s], x[fb][i], 0, 0, 0);
    }
    half8_t phi[2][2];
    den += column_features(x, c.P + kv * kRank + 128 * half, g, phi);
#pragma unroll
    for (int fb = 0; fb < 2; ++fb)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(sS[fb][n][e][lane]), phi[fb][e], acc[n], 0, 0, 0);
  }
  if (token >= T) return;
  float* dst = a.corr + (bh * a.T + token) * kPartStride;
  if (g == 0) dst[0] = den;
#pragma unroll
  for (int n = 0; n < 8; ++n) *reinterpret_cast<float4_t*>(dst + 4 + 16 * n + 4 * g) = acc[n];
}

}  // namespace

int launch_prompt_correction(const ContextCall& a, hipStream_t stream) {
  const int blocks = (a.T + kCorrTokens - 1) / kCorrTokens;
  const dim3 grid((unsigned)((long long)a.cache.B * a.cache.H_q * blocks));
  hipLaunchKernelGGL(prompt_correction_kernel, grid, dim3(64 * kCorrWaves), 0, stream, a, blocks);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
