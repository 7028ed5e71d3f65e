// The linear correction of prompt rows (Sec. 3.2, Eq. 5-6): C_n = phi_q(q) S and C_d = phi_q(q) P of every row, in the rotated basis.
//
// A wave takes 16 NT tokens of one head, both products on v_mfma_f32_16x16x32_f16 and transposed, so that a lane keeps one token
// (column lane % 16) from the logits to the result and nothing goes through LDS:
//   logits^T = W^T q^T: row j of tile i (i = 0..3) of a block of 64 features is feature 4 j + i, so that a lane loads 4 neighbouring features
//              of the 8 channels that it feeds, and its results are 16 neighbouring features, 16 g .. 16 g + 15 (g = lane / 16);
//   C_n^T    = S^T phi^T: those are the positions it feeds, 8 in turn; S from its binary16 tile copy, 4 features in 8 bytes.
// The features are rounded to binary16 (2^-12 of each), as S is; logits, their softmax and the sums are binary32.
// Bound: the weights and the state, 64 KB each, which every wave reads from L2 for 16 NT tokens: 8192 tokens of 32 heads 150 us (0.23 PFLOP/s, 4 % of their call).
#include <hip/hip_runtime.h>

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

__device__ __forceinline__ float column_allmax(float v) {  // over the four lanes of a column
  float x, y;
  pair_across<16>(v, x, y);
  pair_across<32>(fmaxf(x, y), x, y);
  return fmaxf(x, y);
}
__device__ __forceinline__ float column_allsum(float v) {
  float x, y;
  pair_across<16>(v, x, y);
  pair_across<32>(x + y, x, y);
  return x + y;
}

template <int NT>
__global__ __launch_bounds__(256, NT == 1 ? 2 : 1) void prompt_correction_kernel(ContextCall a, long long n_waves, int blocks) {
  const kvlinc_cache& c = a.cache;
  const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
  const long long id = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= n_waves) return;
  const long long bh = id / blocks;  // b H_q + h
  const int i0 = (int)(id - bh * blocks) * 16 * NT, b = (int)(bh / c.H_q), h = (int)(bh - (long long)b * c.H_q);
  const int T = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T;
  if (i0 >= T) return;
  const long long kv = (long long)b * c.H_kv + h / a.gq;

  half8_t q[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint4* src = reinterpret_cast<const uint4*>(a.q + (bh * a.T + min(i0 + 16 * t + j, T - 1)) * kHeadDim) + g;
#pragma unroll
    for (int s = 0; s < 4; ++s) q[t][s] = as_h8(src[4 * s]);  // channels 32 s + 8 g + 0..7
  }
  float4_t acc[NT][8];
  float den[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    den[t] = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[t][n] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    const half_t* W = reinterpret_cast<const half_t*>(c.Wq) + ((long long)h * 2 + half) * kHeadDim * 128;
    float x[NT][2][4][4];  // [64-feature block][tile][row]
#pragma unroll
    for (int fb = 0; fb < 2; ++fb) {
      float4_t d[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[t][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        uint2 w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const uint2*>(W + (32 * s + 8 * g + k) * 128 + 64 * fb + 4 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t r[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t lo = i < 2 ? w[2 * k].x : w[2 * k].y, hi = i < 2 ? w[2 * k + 1].x : w[2 * k + 1].y;
            r[k] = __builtin_amdgcn_perm(hi, lo, (i & 1) == 0 ? 0x05040100u : 0x07060302u);
          }
          const half8_t A = as_h8(make_uint4(r[0], r[1], r[2], r[3]));
#pragma unroll
          for (int t = 0; t < NT; ++t) d[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, q[t][s], d[t][i], 0, 0, 0);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][fb][i][r] = d[t][i][r];
    }
    half8_t phi[NT][2][2];  // [64-feature block][8 of the lane's 16 features]
    const float* P = c.P + kv * kRank + 128 * half;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float m = -INFINITY, z = 0.0f;
#pragma unroll
      for (int fb = 0; fb < 2; ++fb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) m = fmaxf(m, x[t][fb][i][r]);
      m = column_allmax(m);
      float p = 0.0f;
#pragma unroll
      for (int fb = 0; fb < 2; ++fb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 w = *reinterpret_cast<const float4*>(P + 64 * fb + 16 * g + 4 * r);
          const float ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e = __builtin_amdgcn_exp2f((x[t][fb][i][r] - m) * 1.4426950408889634f);
            x[t][fb][i][r] = e;
            z += e;
            p = fmaf(e, ww[i], p);
          }
        }
      const float inv = 1.0f / column_allsum(z);
      den[t] = fmaf(column_allsum(p), inv, den[t]);
#pragma unroll
      for (int fb = 0; fb < 2; ++fb)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          phi[t][fb][e] = as_h8(pack_h2(x[t][fb][0][2 * e] * inv, x[t][fb][1][2 * e] * inv), pack_h2(x[t][fb][2][2 * e] * inv, x[t][fb][3][2 * e] * inv),
                                pack_h2(x[t][fb][0][2 * e + 1] * inv, x[t][fb][1][2 * e + 1] * inv),
                                pack_h2(x[t][fb][2][2 * e + 1] * inv, x[t][fb][3][2 * e + 1] * inv));
    }
    // tile (64-feature block, channel half, 4-feature step) of S16 holds [channel % 64][feature % 4]
    const half_t* S = reinterpret_cast<const half_t*>(c.S16) + kv * (128 * 64 * 4);
#pragma unroll
    for (int fb = 0; fb < 2; ++fb)
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tile = ((2 * half + fb) * 2 + n / 4) * 16 + 4 * g + 2 * e, ch = 16 * (n % 4) + j;
          const uint2 s0 = *reinterpret_cast<const uint2*>(S + (tile * 64 + ch) * 4), s1 = *reinterpret_cast<const uint2*>(S + ((tile + 1) * 64 + ch) * 4);
          const half8_t A = as_h8(make_uint4(s0.x, s0.y, s1.x, s1.y));
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, phi[t][fb][e], acc[t][n], 0, 0, 0);
        }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = i0 + 16 * t + j;
    if (i >= T) continue;
    float* dst = a.corr + (bh * a.T + i) * kPartStride;
    if (g == 0) dst[0] = den[t];
#pragma unroll
    for (int n = 0; n < 8; ++n) *reinterpret_cast<float4_t*>(dst + 4 + 16 * n + 4 * g) = acc[t][n];
  }
}

}  // namespace

int launch_prompt_correction(const ContextCall& a, hipStream_t stream) {
  // 32 tokens a wave share the operands; fewer rows than a wave for every SIMD of the chip that way go by 16.
  const long long heads = (long long)a.cache.B * a.cache.H_q;
  const bool wide = heads * ((a.T + 31) / 32) >= 1024;
  const int blocks = wide ? (a.T + 31) / 32 : (a.T + 15) / 16;
  const long long waves = heads * blocks;
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (wide) hipLaunchKernelGGL(prompt_correction_kernel<2>, grid, dim3(256), 0, stream, a, waves, blocks);
  else hipLaunchKernelGGL(prompt_correction_kernel<1>, grid, dim3(256), 0, stream, a, waves, blocks);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
