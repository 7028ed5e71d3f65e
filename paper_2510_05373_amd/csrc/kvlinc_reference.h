// References of the rows of prompt attention (not part of the C ABI): weights are 2^(score - reference), scores in the log2 domain.
#pragma once

#include "kvlinc_codes.h"

namespace kvlinc {
namespace {

// The reference of a row is its largest score less kHeadroom when it is set, and is set anew when a score passes it by kHeadroom + kLag (most blocks
// only compare): weights stay below 2^13, near 2^8, where the smallest that count are normal binary16 numbers.
constexpr float kHeadroom = 8.0f, kLag = 5.0f;
constexpr float kFusedBound = 0x1p20f;  // references beyond it: no head room, and the exponents are rounded as the reference was
// (a difference: m + 13 is m + 16 where steps are that wide)
__device__ __forceinline__ bool passes(float score, float m) { return score - m > kHeadroom + kLag; }
__device__ __forceinline__ float raised(float score, float m) { return passes(score, m) ? (fabsf(score) > kFusedBound ? score : score - kHeadroom) : m; }
// What the sums so far are multiplied with (0 where nothing was seen).
__device__ __forceinline__ float raised_factor(float m, float to) { return to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - to); }

}  // namespace
}  // namespace kvlinc
