// The correction's features of query rows, phi_q(q) (Sec. 3.2, Eq. 6), on v_mfma_f32_16x16x32_f16, as both kernels that form them take them (not part of
// the C ABI).  A lane keeps one row (column lane % 16 = j) throughout; g = lane / 16.
//   logits^T = W^T q^T: row j of tile i (i = 0..3) of a block of 64 features is feature 4 j + i, so that a lane loads 4 neighbouring features of the
//              8 channels that it feeds, and its results are 16 neighbouring features, 16 g .. 16 g + 15;
//   C_n^T    = S^T phi^T: those are the positions it feeds, 8 in turn; S from its binary16 tile copy, 4 features in 8 bytes.
// The features are rounded to binary16 (2^-12 of each), as S is; logits, their softmax and the sums are binary32.
#pragma once

#include "kvlinc_codes.h"

namespace kvlinc {
namespace {

// Over the four lanes of a column.
__device__ __forceinline__ float column_allmax(float v) {
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

// Operands of the first product, tiles 0..3 of features 64 fb .. 64 fb + 63 and channels 32 s .. 32 s + 31 of one half of a head's weights, [128][128].
__device__ __forceinline__ void weight_operands(const half_t* W, int s, int fb, int j, int g, u32x4_t (&tiles)[4]) {
  u32x2_t w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const u32x2_t*>(W + (32 * s + 8 * g + k) * 128 + 64 * fb + 4 * j);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) tiles[i][k] = __builtin_amdgcn_perm(w[2 * k + 1][i >> 1], w[2 * k][i >> 1], (i & 1) == 0 ? 0x05040100u : 0x07060302u);
}
// Operand of the second: features f .. f + 7 of a channel; tile (64-feature block, channel half, 4-feature step) of S16 holds [channel % 64][feature % 4].
__device__ __forceinline__ u32x4_t state_operand(const half_t* S, int f, int channel) {
  const int tile = ((f >> 6) * 2 + (channel >> 6)) * 16 + ((f & 63) >> 2), ch = channel & 63;
  const u32x2_t a = *reinterpret_cast<const u32x2_t*>(S + (tile * 64 + ch) * 4), b = *reinterpret_cast<const u32x2_t*>(S + ((tile + 1) * 64 + ch) * 4);
  return u32x4_t{a[0], a[1], b[0], b[1]};
}
// The softmax of one half: x[64-feature block][tile], logits, becomes phi[64-feature block][8 of the lane's 16]; returns phi P (P: this half's).
__device__ __forceinline__ float column_features(float4_t (&x)[2][4], const float* P, int g, half8_t (&phi)[2][2]) {
  float m = -INFINITY, z = 0.0f, p = 0.0f;
#pragma unroll
  for (int fb = 0; fb < 2; ++fb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, x[fb][i][r]);
  m = column_allmax(m);
#pragma unroll
  for (int fb = 0; fb < 2; ++fb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float4_t w = *reinterpret_cast<const float4_t*>(P + 64 * fb + 16 * g + 4 * r);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f((x[fb][i][r] - m) * 1.4426950408889634f);
        x[fb][i][r] = e;
        z += e;
        p = fmaf(e, w[i], p);
      }
    }
  const float inv = 1.0f / column_allsum(z);
#pragma unroll
  for (int fb = 0; fb < 2; ++fb)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      phi[fb][e] = as_h8(pack_h2(x[fb][0][2 * e] * inv, x[fb][1][2 * e] * inv), pack_h2(x[fb][2][2 * e] * inv, x[fb][3][2 * e] * inv),
                         pack_h2(x[fb][0][2 * e + 1] * inv, x[fb][1][2 * e + 1] * inv), pack_h2(x[fb][2][2 * e + 1] * inv, x[fb][3][2 * e + 1] * inv));
  return column_allsum(p) * inv;
}

}  // namespace
}  // namespace kvlinc
