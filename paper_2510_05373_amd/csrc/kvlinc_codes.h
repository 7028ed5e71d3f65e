// Packed codes as binary16 numbers, and small pieces shared by the kernels that read the cache with them (not part of the C ABI).
#pragma once

#include "kvlinc_internal.h"
#include "kvlinc_mfma.h"

namespace kvlinc {
namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float2v_t __attribute__((ext_vector_type(2)));

constexpr float kInvSqrtD = 0.08838834764831845f;              // 1 / sqrt(128)
constexpr float kLog2eSqrtD = 1.4426950408889634f * kInvSqrtD;  // scores in the log2 domain: x = q.k log2(e) / sqrt(d)

__device__ __forceinline__ float bits_f32(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ half2_t pack_h2(float a, float b) { return __builtin_convertvector((float2v_t{a, b}), half2_t); }
__device__ __forceinline__ half8_t as_h8(u32x4_t v) { return __builtin_bit_cast(half8_t, v); }
__device__ __forceinline__ half8_t as_h8(uint4 v) { return __builtin_bit_cast(half8_t, v); }
__device__ __forceinline__ half8_t as_h8(half2_t a, half2_t b, half2_t c, half2_t d) {
  return as_h8(make_uint4(as_u32(a), as_u32(b), as_u32(c), as_u32(d)));
}

// A packed word holds the bit pairs of two codes in every nibble, so that the bits of one of them, with the nibble's other two bits
// set to 0 and 1, are the FP4 (E2M1) number code - 1.5: `first` takes the codes p = 0, 2, ..., 14 of the word, `second` the odd ones.
struct Nibbles {
  uint32_t first, second;
};
__device__ __forceinline__ uint32_t code_bits() {
  uint32_t m = 0xAAAAAAAAu;
  asm("" : "+s"(m));  // (opaque, so that taking the code's bits and setting the others is one bit-field insert)
  return m;
}
__device__ __forceinline__ Nibbles nibbles_of(uint32_t w) {
  const uint32_t m = code_bits();
  return Nibbles{0x11111111u ^ (m & (w ^ 0x11111111u)), 0x11111111u ^ (m & ((w << 1) ^ 0x11111111u))};
}
// Byte SEL of such nibbles, two codes, as binary16: (code - 1.5) scale, scale a power of two.  One instruction, exact.
template <int SEL>
__device__ __forceinline__ half2_t nibble_pair(uint32_t nibbles, float scale) {
  return __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(nibbles, scale, SEL));
}
// The same for codes of BITS bits, code - Rec<BITS>::kCentre: of 4 bits, the high digit's pair times 4 plus the low digit's (exact).
template <int BITS, int SEL>
__device__ __forceinline__ half2_t code_pair(const uint32_t (&plane)[BITS / 2], float scale) {
  if constexpr (BITS == 2) return nibble_pair<SEL>(plane[0], scale);
  else return nibble_pair<SEL>(plane[0], 4.0f * scale) + nibble_pair<SEL>(plane[1], scale);
}

// Eight numbers over a scale, a power of two, as FP4 (E2M1) ones, the first in the lowest bits; a tie goes to the even one.
__device__ __forceinline__ uint32_t fp4_of(const float (&v)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

// Exponent (biased by 127) of a scale for what the rounding to binary16 leaves of numbers up to one of these bits: half a step of it is
// 2^(field - 26), 4 of the scale.
__device__ __forceinline__ uint32_t low_scale_of(uint32_t largest) { return max(largest >> 10, 1u) + 99u; }

// Butterflies between the 16 lanes of a DPP row, strides 1, 2, 4, 8, NV vectors at once.
template <int NV>
__device__ __forceinline__ void row16_butterflies(float (&v)[NV], int lane) {
  auto sign = [&](int bit) { return (lane & bit) != 0 ? -1.0f : 1.0f; };
  const float s1 = sign(1), s2 = sign(2), s4 = sign(4), s8 = sign(8);
#pragma unroll
  for (int u = 0; u < NV; ++u) v[u] = __builtin_fmaf(v[u], s1, dpp_f<kQuadSwap1>(v[u]));
#pragma unroll
  for (int u = 0; u < NV; ++u) v[u] = __builtin_fmaf(v[u], s2, dpp_f<kQuadSwap2>(v[u]));
#pragma unroll
  for (int u = 0; u < NV; ++u) v[u] = __builtin_fmaf(v[u], s4, dpp_f<kQuadMirror>(dpp_f<kRowHalfMirror>(v[u])));
#pragma unroll
  for (int u = 0; u < NV; ++u) v[u] = __builtin_fmaf(v[u], s8, dpp_f<kRowRor8>(v[u]));
}
// Three butterfly stages over 8 neighbouring channels of a lane.
__device__ __forceinline__ void lane8_butterflies(float (&v)[8]) {
#pragma unroll
  for (int h = 1; h < 8; h *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & h) == 0) {
        const float a = v[i], b = v[i + h];
        v[i] = a + b;
        v[i + h] = a - b;
      }
}

// Softmax sums relative to 2^m (m: log2 domain) and the correction, e^0 terms, in one quotient: (den + 2^-m C_d), both sides times 2^m, but by no
// less than 2^-64: the sums count some token as 1 or more, C_d and C_n stay in range under 2^64, so the divisor is a normal number however little is
// added.  Where nothing is added (C_d = 0: no quantized token yet) the factor cancels and is left out.  (Times 2^min(m, 0) the sums vanished for
// rows whose logits are all below -82, and 0 / 0 was left.)
struct Shares {
  float softmax, correction;  // factors
};
__device__ __forceinline__ Shares shares_of(float m, float c_d) {
  const float to = fmaxf(m, -64.0f);
  return Shares{c_d != 0.0f ? __builtin_amdgcn_exp2f(m - to) : 1.0f, __builtin_amdgcn_exp2f(-to)};
}

// Bits 15 and 31: the halves of a word that are infinite or not a number; and the word with zeros in their places.  A value that a row does not see
// must not reach it, and 0 times such a value is not a number.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t w) { return w & ~((not_finite(w) >> 15) * 0xffffu); }

// Reference of a row as the others' parts are joined with it: that of a row whose scores are not numbers was never set (a maximum passes them by), and
// -inf would leave its sum out.
__device__ __forceinline__ float reference_of(float m, float l) { return l != l && m == -INFINITY ? 0.0f : m; }

// What a query sees: its position p, the window's first token, the sinks.  Token t <= p is seen if t >= low or t < sinks.
__device__ __forceinline__ int window_low(int p, int window) { return window > 0 ? max(p - window + 1, 0) : 0; }

// Counters of a sequence, kept inside the cache's storage.
struct Lengths {
  int nq, nr;
  __device__ __forceinline__ int total() const { return nq + nr; }
  __device__ __forceinline__ int groups() const { return (nq + kGroup - 1) / kGroup; }
};
__device__ __forceinline__ Lengths lengths_of(const kvlinc_cache& c, int b) {
  const long long cap = c.max_groups * kGroup;
  return Lengths{(int)min((long long)max(c.n_quant[b], 0), cap), min(max(c.n_res[b], 0), c.R)};
}

}  // namespace
}  // namespace kvlinc
