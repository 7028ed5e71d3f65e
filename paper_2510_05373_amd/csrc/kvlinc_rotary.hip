// Rotary positions of new rows: queries and keys turned, values taken along, from any strides to the layout of the cache's calls.
//
// A wave has one token; 8 lanes have a row of 128 numbers, so that it takes 8 heads at a time, `steps` times.  A lane has the same pairs in every
// row: it forms its 8 sines and cosines once.  The angle in turns, p freq / 2 pi, is formed in binary64 and reduced there to a quarter of a turn around
// its nearest one (exact), so that binary32 has nothing to lose at far positions; sine and cosine of |x| <= pi / 4 are their Taylor series up to
// x^9 and x^10 (the next terms are below 2^-29).
// Bound: bytes, a row in and out once.
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_codes.h"

namespace kvlinc {
namespace {

typedef __bf16 bf16_t;
constexpr int kRotaryWaves = 4;

// Which numbers of a row a lane has, two runs of 8: kApart, kNeighbours: pairs within the lane.  kAny: pairs `channels` / 2 apart where that is
// not a multiple of 8; the partners come through LDS.
enum Layout { kApart, kNeighbours, kAny };

struct Turn {
  float cos, sin;
};
__device__ __forceinline__ Turn turn_of(double position, double freq, float magnitude) {
  const double turns = position * (freq * 0.15915494309189533577);  // 1 / (2 pi)
  const double quarters = 4.0 * (turns - __builtin_rint(turns)), nearest = __builtin_rint(quarters);
  const int k = (int)nearest & 3;
  const float x = (float)(quarters - nearest) * 1.57079632679489662f, z = x * x;
  const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
  const float cos = (k & 1) != 0 ? s : c, sin = (k & 1) != 0 ? c : s;
  return Turn{(((k + 1) & 2) != 0 ? -cos : cos) * magnitude, ((k & 2) != 0 ? -sin : sin) * magnitude};
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  typedef T run_t __attribute__((ext_vector_type(8)));
  const run_t x = *reinterpret_cast<const run_t*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  typedef T run_t __attribute__((ext_vector_type(8)));
  run_t x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
  *reinterpret_cast<run_t*>(p) = x;
}

// Grid: tokens by kRotaryWaves (and sequences) in x, runs of 8 `steps` heads in y.
template <Layout L, typename IN, typename OUT>
__global__ __launch_bounds__(64 * kRotaryWaves) void rotary_kernel(RotaryCall a) {
  constexpr int kPartners = L == kAny ? 16 : 8;  // angles of a lane
  __shared__ float sRow[L == kAny ? kRotaryWaves : 1][8][L == kAny ? kHeadDim + 4 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 7;
  const uint32_t place = blockIdx.x * kRotaryWaves + wave;  // (sequence, token)
  const int b = (int)(place / (uint32_t)a.T), t = (int)(place - (uint32_t)b * a.T);
  if (b >= a.B) return;
  if (a.n_new != nullptr && t >= a.n_new[b]) return;
  long long p = a.depth != nullptr ? a.depth[place] : t;
  if (a.n_quant != nullptr) p += (long long)a.n_quant[b] + a.n_res[b];
  if (a.first != nullptr) p += a.first[b];
  const double position = (double)p;

  // the lane's runs at[0], at[1] of 8 channels
  const int half = a.channels / 2;
  const bool turned = L != kApart || l < half / 8;
  const int rest = a.channels + 16 * (l - half / 8);
  const int at[2] = {L == kApart ? (turned ? 8 * l : rest) : 16 * l, L == kApart ? (turned ? half + 8 * l : rest + 8) : 16 * l + 8};
  Turn turn[kPartners];
#pragma unroll
  for (int i = 0; i < kPartners; ++i) {
    const int c = 16 * l + i, pair = L == kAny ? (c < half ? c : c - half) : 8 * l + i;
    turn[i] = turn_of(position, a.freq[min(pair, half - 1)], a.magnitude);
  }

  for (int step = 0; step < a.steps; ++step) {
    const int row = ((int)blockIdx.y * a.steps + step) * 8 + (lane >> 3);
    if (row >= a.heads) break;  // (the lanes of a row go together)
    const int h1 = row - a.rows[0].heads, h2 = h1 - a.rows[1].heads, which = h1 < 0 ? 0 : h2 < 0 ? 1 : 2, h = h1 < 0 ? row : h2 < 0 ? h1 : h2;
    const auto of_row = [&](auto q, auto k, auto v) { return which == 0 ? q : which == 1 ? k : v; };
    const auto& [q, k, v] = a.rows;
    const IN* in = static_cast<const IN*>(of_row(q.in, k.in, v.in)) + of_row(b * q.sequence_stride + t * q.token_stride, b * k.sequence_stride + t * k.token_stride, b * v.sequence_stride + t * v.token_stride) +
                   h * of_row(q.head_stride, k.head_stride, v.head_stride);
    OUT* out = static_cast<OUT*>(of_row(q.out, k.out, v.out)) + (((long long)b * of_row(q.heads, k.heads, v.heads) + h) * a.T + t) * kHeadDim;
    float x[2][8], y[2][8];
    load8(in + at[0], x[0]);
    load8(in + at[1], x[1]);
    if constexpr (L == kApart) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[0][i] = fmaf(x[0][i], turn[i].cos, -x[1][i] * turn[i].sin);
        y[1][i] = fmaf(x[0][i], turn[i].sin, x[1][i] * turn[i].cos);
      }
    } else if constexpr (L == kNeighbours) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[i / 4][2 * (i % 4)], v = x[i / 4][2 * (i % 4) + 1];
        const bool is = 8 * l + i < half;
        y[i / 4][2 * (i % 4)] = is ? fmaf(u, turn[i].cos, -v * turn[i].sin) : u;
        y[i / 4][2 * (i % 4) + 1] = is ? fmaf(u, turn[i].sin, v * turn[i].cos) : v;
      }
    } else {
      float* mine = sRow[wave][lane >> 3];
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[16 * l + i] = x[i / 8][i % 8];
      wave_order();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = 16 * l + i;
        const float other = mine[c < half ? c + half : c < a.channels ? c - half : c], own = x[i / 8][i % 8];
        const float part = other * turn[i].sin;
        y[i / 8][i % 8] = c >= a.channels ? own : fmaf(own, turn[i].cos, c < half ? -part : part);
      }
      wave_order();
    }
    const bool pass = which == 2 || !turned;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i / 8][i % 8] = pass ? x[i / 8][i % 8] : y[i / 8][i % 8];
    store8(out + at[0], y[0]);
    store8(out + at[1], y[1]);
  }
}

template <Layout L, typename IN>
void launch_to(const RotaryCall& a, int dtype_out, dim3 grid, hipStream_t stream) {
  const dim3 block(64 * kRotaryWaves);
  if (dtype_out == KVLINC_F16) hipLaunchKernelGGL((rotary_kernel<L, IN, half_t>), grid, block, 0, stream, a);
  else if (dtype_out == KVLINC_BF16) hipLaunchKernelGGL((rotary_kernel<L, IN, bf16_t>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<L, IN, float>), grid, block, 0, stream, a);
}
template <Layout L>
void launch_layout(const RotaryCall& a, int dtype_in, int dtype_out, dim3 grid, hipStream_t stream) {
  if (dtype_in == KVLINC_F16) launch_to<L, half_t>(a, dtype_out, grid, stream);
  else if (dtype_in == KVLINC_BF16) launch_to<L, bf16_t>(a, dtype_out, grid, stream);
  else launch_to<L, float>(a, dtype_out, grid, stream);
}

}  // namespace

int launch_rotary(const RotaryCall& call, bool interleaved, int dtype_in, int dtype_out, hipStream_t stream) {
  RotaryCall a = call;
  const long long tokens = (long long)a.B * a.T, runs = (a.heads + 7) / 8;
  // heads of a token are shared out among waves until there are some 2048 of them
  long long shares = 2048 / tokens;
  if (shares > runs) shares = runs;
  if (shares < 1) shares = 1;
  a.steps = (int)((runs + shares - 1) / shares);
  const dim3 grid((unsigned)((tokens + kRotaryWaves - 1) / kRotaryWaves), (unsigned)((runs + a.steps - 1) / a.steps));
  if (interleaved) launch_layout<kNeighbours>(a, dtype_in, dtype_out, grid, stream);
  else if (a.channels % 16 == 0) launch_layout<kApart>(a, dtype_in, dtype_out, grid, stream);
  else launch_layout<kAny>(a, dtype_in, dtype_out, grid, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
