// Rotary positions of new rows: queries and keys turned, values taken along, from any strides to the layout of the cache's calls.
//
// A wave has one token; 8 lanes have a row of 128 numbers, so that it takes 8 heads at a time, `steps` times.  A lane has the same pairs in every
// row: it forms its 8 sines and cosines once.  The angle in turns, p freq / 2 pi, is formed in binary64 (the constant and two products: 2.56 * 2^-53 of it at
// most) and reduced there to a quarter of a turn around its nearest one (exact), so that binary32 has nothing to lose at far positions; sine and cosine of
// |x| <= pi / 4 are their Taylor series up to x^9 and x^10 (the next terms are below 2^-29).
// Bound: bytes, a row in and out once: 16 sequences of up to 2048 tokens, 48 heads, binary16 from bfloat16: 109.7 us, 5.4 TB/s; single tokens and drafts: the
// host's call, 9.7 us, of which the kernel takes 3.6 and 5.
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_codes.h"

namespace kvlinc {
namespace {

typedef __bf16 bf16_t;
constexpr int kRotaryWaves = 4;
// Loads and stores past the caches from so many bytes of results on (the caches next to the XCDs hold 32 MB in all): 96 MB of binary16 42.4 -> 38.9 us, 48 MB
// 22.2 -> 20.9; not from 2 bytes a number to 4, where a row's lanes read 64 bytes at a time: 132 -> 144.
constexpr long long kStreamedBytes = 64ll << 20;

// Which numbers of a row a lane has: 16 / RUN runs of RUN, so that the 8 lanes of a row have 128 bytes side by side of the wider type: RUN = 8, or 4 with
// binary32.  (With binary32 in runs of 8, and with pairs of neighbours in runs of 8 beside each other, a store left every second 16 bytes to the next one:
// 384 MB of binary32 185 us for 132, 192 MB of neighbours 91 for 72.)
// kApart, kNeighbours: pairs within the lane.  kAny: pairs `channels` / 2 apart, the partners come through LDS.
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

template <int RUN, bool STREAMED, typename T>
__device__ __forceinline__ void load_run(const T* p, float* v) {
  typedef T run_t __attribute__((ext_vector_type(RUN)));
  run_t x;
  if constexpr (STREAMED) x = __builtin_nontemporal_load(reinterpret_cast<const run_t*>(p));
  else x = *reinterpret_cast<const run_t*>(p);
#pragma unroll
  for (int i = 0; i < RUN; ++i) v[i] = (float)x[i];
}
template <int RUN, bool STREAMED, typename T>
__device__ __forceinline__ void store_run(T* p, const float* v) {
  typedef T run_t __attribute__((ext_vector_type(RUN)));
  run_t x;
#pragma unroll
  for (int i = 0; i < RUN; ++i) x[i] = (T)v[i];
  if constexpr (STREAMED) __builtin_nontemporal_store(x, reinterpret_cast<run_t*>(p));
  else *reinterpret_cast<run_t*>(p) = x;
}

// Grid: tokens by kRotaryWaves (and sequences) in x, runs of 8 `steps` heads in y.
template <Layout L, bool STREAMED, typename IN, typename OUT>
__global__ __launch_bounds__(64 * kRotaryWaves) void rotary_kernel(RotaryCall a) {
  constexpr int kAngles = L == kAny ? 16 : 8;  // of a lane
  constexpr int RUN = sizeof(IN) == 4 || sizeof(OUT) == 4 ? 4 : 8, RUNS = 16 / RUN;
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

  // the lane's runs; kApart: runs 2 p and 2 p + 1 have the two halves of pairs, or (not turned[p]) channels behind those that turn
  const int half = a.channels / 2;
  int at[RUNS];
  bool turned[RUNS / 2];
#pragma unroll
  for (int r = 0; r < RUNS; ++r) {
    const int j = l + 8 * (r / 2), beyond = RUN * j - half, second = r % 2;
    if (second == 0) turned[r / 2] = L != kApart || beyond < 0;
    at[r] = L != kApart ? RUN * (l + 8 * r) : beyond < 0 ? RUN * j + second * half : a.channels + beyond + second * (kHeadDim / 2 - half);
  }
  Turn turn[kAngles];
#pragma unroll
  for (int i = 0; i < kAngles; ++i) {
    const int c = L == kApart ? at[2 * (i / RUN)] + i % RUN : L == kNeighbours ? at[2 * i / RUN] + 2 * i % RUN : at[i / RUN] + i % RUN;
    const int pair = L == kNeighbours ? c / 2 : L == kAny && c >= half ? c - half : c;
    turn[i] = turn_of(position, a.freq[min(pair, half - 1)], a.magnitude);
    if (L == kAny) turn[i] = c < half ? Turn{turn[i].cos, -turn[i].sin} : Turn{turn[i].sin, turn[i].cos};  // of the pair's first number, and its second
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
    float x[16], y[16];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) load_run<RUN, STREAMED>(in + at[r], x + r * RUN);
    if constexpr (L == kApart) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int u = 2 * (i / RUN) * RUN + i % RUN, v = u + RUN;
        y[u] = fmaf(x[u], turn[i].cos, -x[v] * turn[i].sin);
        y[v] = fmaf(x[u], turn[i].sin, x[v] * turn[i].cos);
      }
    } else if constexpr (L == kNeighbours) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[2 * i], v = x[2 * i + 1];
        const bool is = at[2 * i / RUN] + 2 * i % RUN < a.channels;
        y[2 * i] = is ? fmaf(u, turn[i].cos, -v * turn[i].sin) : u;
        y[2 * i + 1] = is ? fmaf(u, turn[i].sin, v * turn[i].cos) : v;
      }
    } else {
      float* mine = sRow[wave][lane >> 3];
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[at[i / RUN] + i % RUN] = x[i];
      wave_order();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = at[i / RUN] + i % RUN;
        const float other = mine[c < half ? c + half : c < a.channels ? c - half : c], u = c < half ? x[i] : other, v = c < half ? other : x[i];
        y[i] = c >= a.channels ? x[i] : fmaf(u, turn[i].cos, v * turn[i].sin);
      }
      wave_order();
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = which == 2 || !turned[i / (2 * RUN)] ? x[i] : y[i];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) store_run<RUN, STREAMED>(out + at[r], y + r * RUN);
  }
}

template <Layout L, bool STREAMED, typename IN>
void launch_to(const RotaryCall& a, int dtype_out, dim3 grid, hipStream_t stream) {
  const dim3 block(64 * kRotaryWaves);
  if (dtype_out == KVLINC_F16) hipLaunchKernelGGL((rotary_kernel<L, STREAMED, IN, half_t>), grid, block, 0, stream, a);
  else if (dtype_out == KVLINC_BF16) hipLaunchKernelGGL((rotary_kernel<L, STREAMED, IN, bf16_t>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<L, STREAMED, IN, float>), grid, block, 0, stream, a);
}
template <Layout L, bool STREAMED>
void launch_from(const RotaryCall& a, int dtype_in, int dtype_out, dim3 grid, hipStream_t stream) {
  if (dtype_in == KVLINC_F16) launch_to<L, STREAMED, half_t>(a, dtype_out, grid, stream);
  else if (dtype_in == KVLINC_BF16) launch_to<L, STREAMED, bf16_t>(a, dtype_out, grid, stream);
  else launch_to<L, STREAMED, float>(a, dtype_out, grid, stream);
}
template <Layout L>
void launch_layout(const RotaryCall& a, int dtype_in, int dtype_out, bool streamed, dim3 grid, hipStream_t stream) {
  if (streamed) launch_from<L, true>(a, dtype_in, dtype_out, grid, stream);
  else launch_from<L, false>(a, dtype_in, dtype_out, grid, stream);
}

}  // namespace

int launch_rotary(const RotaryCall& call, bool interleaved, int dtype_in, int dtype_out, hipStream_t stream) {
  RotaryCall a = call;
  const long long tokens = (long long)a.B * a.T, runs = (a.heads + 7) / 8;
  // heads of a token are shared out among waves until there are some 2048 of them (512, 1024, 2048, 4096: 512 tokens of 48 heads 5.8, 4.7, 4.8, 5.1 us;
  // 1024 of 96 heads 12.8, 12.7, 10.6, 11.0)
  long long shares = 2048 / tokens;
  if (shares > runs) shares = runs;
  if (shares < 1) shares = 1;
  a.steps = (int)((runs + shares - 1) / shares);
  const dim3 grid((unsigned)((tokens + kRotaryWaves - 1) / kRotaryWaves), (unsigned)((runs + a.steps - 1) / a.steps));
  const bool streamed = tokens * a.heads * kHeadDim * (dtype_out == KVLINC_F32 ? 4 : 2) >= kStreamedBytes && (dtype_in == KVLINC_F32 || dtype_out != KVLINC_F32);
  // Where a part of the channels turns, a lane with the two halves of its pairs leaves less than 128 bytes side by side: 8 x 2048 tokens of 48 heads, 32, 64
  // and 96 channels 84, 83 and 85 us, past the caches 109, 90 and 109; with runs side by side, the partners by LDS, and past the caches 75, 76 and 79, but
  // 2 x 1024 tokens 15.8 for 11.9 (twice the angles).
  const bool apart = a.channels == kHeadDim || (a.channels % 16 == 0 && !streamed);
  if (interleaved) launch_layout<kNeighbours>(a, dtype_in, dtype_out, streamed, grid, stream);
  else if (apart) launch_layout<kApart>(a, dtype_in, dtype_out, streamed, grid, stream);
  else launch_layout<kAny>(a, dtype_in, dtype_out, streamed, grid, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
