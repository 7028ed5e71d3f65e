// Reading the cache back: keys and values of a range of tokens, dequantized.
//
// A workgroup takes the tokens of one aligned block of 128 positions of a (sequence, KV head), keys or values: packed ones from the block's
// record, raw ones from the window (a cache with a partial last group has both in one block).
// Values are rotated back by butterflies on the codes themselves: H (s c + z) = s (H c) + z H 1, and the sums of 128 centred
// codes, multiples of 1/2 below 1024, are exact in binary16, two tokens an instruction.  H 1 = sqrt(128) e_0 leaves the zero-point to channel 0.
// So a number is rounded once in binary32 and once to its type.  Bound: bytes written (256 to 512 a token and tensor against 32 to 64
// read); rows go through LDS so that a wave stores whole lines.
// 16 sequences of 8k tokens, 8 heads, 2 bits: binary16 and bfloat16 138 us, rotated 133, binary32 209 (5.5 TB/s), rotated 198; 4 bits 145.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

struct BF16 { uint16_t bits; };
template <typename OUT>
__device__ __forceinline__ OUT rounded(float v);
template <>
__device__ __forceinline__ float rounded<float>(float v) { return v; }
template <>
__device__ __forceinline__ half_t rounded<half_t>(float v) { return (half_t)fminf(fmaxf(v, -65504.0f), 65504.0f); }
template <>
__device__ __forceinline__ BF16 rounded<BF16>(float v) {  // to nearest even (finite numbers)
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  return BF16{(uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16)};
}

// 16 rows of a wave in LDS, 16 bytes more than a row apart; a wave fills and stores them twice for its 32 tokens (twice the rows: half the
// workgroups on a compute unit).
constexpr int kRowsHeld = 16;
template <typename OUT>
struct WaveRows {
  static constexpr int kStride = kHeadDim + 16 / sizeof(OUT);
  OUT x[kRowsHeld][kStride];
};
// Where rows go: those of positions from .. to - 1.  Stores past the caches: a large range written through them takes nearly twice as long (16
// sequences of 8k tokens, 8 heads: 246 us, 140 so), and rows that the next launch reads (kvlinc_dense.hip) are read no slower.
template <typename OUT>
struct Target {
  OUT* out;
  long long first;
  int from, to, at;  // at: position of the block
};
template <typename OUT, typename F>
__device__ __forceinline__ void store_rows(const WaveRows<OUT>& rows, const Target<OUT>& d, int lane, F token_of) {  // token_of(r): of row r, in the block
  constexpr int kLanes = kHeadDim * sizeof(OUT) / 16;  // lanes a row takes, 16 bytes each
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS instructions stay in order)
#pragma unroll
  for (int r0 = 0; r0 < kRowsHeld; r0 += 64 / kLanes) {
    const int r = r0 + lane / kLanes, t = d.at + token_of(r);
    if (t < d.from || t >= d.to) continue;
    const u32x4_t v = reinterpret_cast<const u32x4_t*>(&rows.x[r][0])[lane % kLanes];
    u32x4_t* dst = reinterpret_cast<u32x4_t*>(d.out + (t - d.first) * kHeadDim) + lane % kLanes;
    __builtin_nontemporal_store(v, dst);
  }
  __builtin_amdgcn_wave_barrier();
}

template <int BITS, int SEL>
__device__ __forceinline__ void key_pairs(const uint32_t (&e)[BITS / 2], const uint32_t (&s)[16], const uint32_t (&z)[16], int at, float (&v)[8]) {
  const half2_t c = code_pair<BITS, SEL>(e, 1.0f), ss = as_h2(s[at + SEL]), zz = as_h2(z[at + SEL]);
#pragma unroll
  for (int i = 0; i < 2; ++i) v[2 * SEL + i] = fmaf((float)ss[i], (float)c[i] + Rec<BITS>::kCentre, (float)zz[i]);
}

// Where what the rounding of keys leaves goes, or NULL: rows as those of the keys, see low_scores.
struct LowTarget {
  u32x4_t* rows;  // [4]
  uint32_t* scale;
};

// Keys: wave w has tokens 32 w .. 32 w + 31; a lane two of them, 32 channels each.
template <int BITS, typename OUT, bool LOW>
__device__ __forceinline__ void read_keys(const uint32_t* rec, WaveRows<OUT>& rows, const Target<OUT>& to, const LowTarget& low, int wave, int lane) {
  const int j = lane & 15, g = lane >> 4;
  uint32_t s[16], z[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 a = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kKeyScale)[4 * g + i], b = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kKeyZero)[4 * g + i];
    s[4 * i] = a.x; s[4 * i + 1] = a.y; s[4 * i + 2] = a.z; s[4 * i + 3] = a.w;
    z[4 * i] = b.x; z[4 * i + 1] = b.y; z[4 * i + 2] = b.z; z[4 * i + 3] = b.w;
  }
  uint32_t scale = 0;  // of this lane's 32 channels, for the whole group
  if constexpr (LOW) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const half_t levels = (half_t)(float)Rec<BITS>::kLevels;
      const uint32_t lowest = z[i] & 0x7fff7fffu, highest = as_u32(__builtin_elementwise_fma(as_h2(s[i]), half2_t{levels, levels}, as_h2(z[i]))) & 0x7fff7fffu;
      top = max(top, max(max(lowest & 0xffffu, lowest >> 16), max(highest & 0xffffu, highest >> 16)));
    }
    scale = low_scale_of(top);
  }
  u32x4_t rest = {0, 0, 0, 0};
  uint4 w[BITS / 2];
#pragma unroll
  for (int pl = 0; pl < BITS / 2; ++pl) w[pl] = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kKeyTile + 1024 * pl)[64 * wave + lane];
#pragma unroll
  for (int q = 0; q < 4; ++q) {  // token 16 (q / 2) + j of the wave's, channels 32 g + 16 (q % 2) + 0..15
    uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles n = nibbles_of(q == 0 ? w[pl].x : q == 1 ? w[pl].y : q == 2 ? w[pl].z : w[pl].w);
      e[pl] = n.first; o[pl] = n.second;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float v[8];
      const int at = 8 * (q % 2) + 4 * u;
      if (u == 0) { key_pairs<BITS, 0>(e, s, z, at, v); key_pairs<BITS, 1>(e, s, z, at, v); key_pairs<BITS, 2>(e, s, z, at, v); key_pairs<BITS, 3>(e, s, z, at, v); }
      else { key_pairs<BITS, 0>(o, s, z, at, v); key_pairs<BITS, 1>(o, s, z, at, v); key_pairs<BITS, 2>(o, s, z, at, v); key_pairs<BITS, 3>(o, s, z, at, v); }
      OUT* dst = &rows.x[j][32 * g + 16 * (q % 2) + 8 * u];
#pragma unroll
      for (int i = 0; i < 8; ++i) dst[i] = rounded<OUT>(v[i]);
      if constexpr (LOW) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= (float)rounded<half_t>(v[i]);
        rest[2 * (q % 2) + u] = fp4_of(v, bits_f32(scale << 23));
      }
    }
    if constexpr (LOW) {
      const int t = to.at + 32 * wave + 16 * (q / 2) + j;
      if (q % 2 == 1 && t >= to.from && t < to.to) {
        __builtin_nontemporal_store(rest, low.rows + (t - to.first) * 4 + g);
        reinterpret_cast<uint8_t*>(low.scale + (t - to.first))[g] = (uint8_t)scale;
      }
    }
    if (q % 2 == 1) store_rows<OUT>(rows, to, lane, [&](int r) { return 32 * wave + 16 * (q / 2) + r; });
  }
}

__device__ __forceinline__ half2_t dpp_h2_swap(half2_t v, int stage) {
  const uint32_t u = as_u32(v);
  return as_h2(stage == 0 ? dpp_u<kQuadSwap1>(u) : stage == 1 ? dpp_u<kQuadSwap2>(u) : stage == 2 ? dpp_u<kQuadMirror>(dpp_u<kRowHalfMirror>(u)) : dpp_u<kRowRor8>(u));
}
// Butterflies over the channels 32 u + 16 n + j (u = lane / 16, n = 0, 1, j = lane % 16) of two tokens.
__device__ __forceinline__ void rotate_codes(half2_t (&v)[2], int lane) {
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    const half_t one = (half_t)((lane >> st) & 1 ? -1.0f : 1.0f);
#pragma unroll
    for (int n = 0; n < 2; ++n) v[n] = __builtin_elementwise_fma(v[n], half2_t{one, one}, dpp_h2_swap(v[n], st));
  }
  const half2_t a = v[0] + v[1], b = v[0] - v[1];
  v[0] = a; v[1] = b;
  const half_t s16 = (half_t)((lane & 16) ? -1.0f : 1.0f), s32 = (half_t)((lane & 32) ? -1.0f : 1.0f);
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const auto x = __builtin_amdgcn_permlane16_swap(as_u32(v[n]), as_u32(v[n]), false, false);
    v[n] = __builtin_elementwise_fma(as_h2(x[1]), half2_t{s16, s16}, as_h2(x[0]));
    const auto y = __builtin_amdgcn_permlane32_swap(as_u32(v[n]), as_u32(v[n]), false, false);
    v[n] = __builtin_elementwise_fma(as_h2(y[1]), half2_t{s32, s32}, as_h2(y[0]));
  }
}

// Values: wave w has tokens 16 i + 4 w + 0..3 (i = 0..7), two of the four (t) at a time, row 2 i + t % 2 of its rows; a lane channels 32 u + 16 n + j of all of them.
template <int BITS, typename OUT, bool ROTATED, int SEL>
__device__ __forceinline__ void value_pairs(const uint32_t (&e)[2][BITS / 2], const uint32_t* sz, int t, WaveRows<OUT>& rows, int lane) {
  const int j = lane & 15, u = lane >> 4;
  half2_t c[2] = {code_pair<BITS, SEL>(e[0], 1.0f), code_pair<BITS, SEL>(e[1], 1.0f)};
  if constexpr (!ROTATED) rotate_codes(c, lane);
#pragma unroll
  for (int k = 0; k < 2; ++k) {  // token 16 i + 4 w + t, i = 2 SEL + k
    const half2_t p = as_h2(sz[2 * SEL + k]);
    const float s = (float)p[0], mid = fmaf(s, Rec<BITS>::kCentre, (float)p[1]);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float x = (float)c[n][k];
      float v;
      if constexpr (ROTATED) v = fmaf(s, x + Rec<BITS>::kCentre, (float)p[1]);
      else v = fmaf(s, x, n == 0 && lane == 0 ? 128.0f * mid : 0.0f) * kInvSqrtD;
      rows.x[2 * (2 * SEL + k) + (t & 1)][32 * u + 16 * n + j] = rounded<OUT>(v);
    }
  }
}
template <int BITS, typename OUT, bool ROTATED>
__device__ __forceinline__ void read_values(const uint32_t* rec, WaveRows<OUT>& rows, const Target<OUT>& to, int wave, int lane) {
  const int j = lane & 15, u = lane >> 4;
#pragma unroll
  for (int hg = 0; hg < 2; ++hg) {
    const int g = (wave >> 1) + 2 * hg, w = wave & 1;
    uint32_t words[2][BITS / 2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int pl = 0; pl < BITS / 2; ++pl) words[n][pl] = rec[Rec<BITS>::kValueTile + 1024 * pl + (64 * u + j + 16 * g) * 4 + 2 * n + w];
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      uint32_t e[2][BITS / 2];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int pl = 0; pl < BITS / 2; ++pl) {
          const Nibbles nb = nibbles_of(words[n][pl]);
          e[n][pl] = odd ? nb.second : nb.first;
        }
      const int t = 2 * hg + odd;
      const uint4* src = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kValueSZ) + 2 * (4 * wave + t);
      const uint4 a = src[0], b = src[1];
      const uint32_t sz[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      value_pairs<BITS, OUT, ROTATED, 0>(e, sz, t, rows, lane);
      value_pairs<BITS, OUT, ROTATED, 1>(e, sz, t, rows, lane);
      value_pairs<BITS, OUT, ROTATED, 2>(e, sz, t, rows, lane);
      value_pairs<BITS, OUT, ROTATED, 3>(e, sz, t, rows, lane);
    }
    store_rows<OUT>(rows, to, lane, [&](int r) { return 16 * (r >> 1) + 4 * wave + 2 * hg + (r & 1); });
  }
}

// Grid, one-dimensional: block of 128 positions fastest, then (sequence, KV head); keys in the first half, values in the second (one
// half where one of the two is not asked for).
struct ReadRange {
  const int32_t* first_of;  // first token of each sequence; NULL: window_base(tokens, window)
  int window, T;            // T rows
  int lead, lead_blocks;    // ahead of them: the first `lead` tokens, blocks of 128 of those
  long long pair_rows;      // rows from one (sequence, KV head) to the next
  int blocks, per_tensor;
  LowTarget low;
};
// Workgroups are dealt to the 8 XCDs in turn; runs of 64 blocks (2 MB of binary16 rows) go to one of them, so that each writes few pages at a time:
// 16 sequences of 8k tokens, 8 heads, outputs and records that no cache holds: 197 us without, 163 with runs of 16, 144 of 32, 142 of 64, 139 of 128
// (longer runs share a batch of few sequences out less evenly).
__device__ __forceinline__ int in_runs(int id, int all) {
  constexpr int kRun = 64;
  const int y = id >> 3, run = y / kRun;
  return id < all - all % (8 * kRun) ? (run * 8 + (id & 7)) * kRun + (y - run * kRun) : id;
}
template <int BITS, typename OUT, bool ROTATED, bool LOW>
__global__ __launch_bounds__(256) void read_kernel(kvlinc_cache c, ReadRange range, OUT* k_out, OUT* v_out) {
  const int blocks = range.blocks, per_tensor = range.per_tensor;
  __shared__ __align__(16) WaveRows<OUT> all[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool values = k_out == nullptr || (int)blockIdx.x >= per_tensor;
  const int id = in_runs((int)blockIdx.x >= per_tensor ? blockIdx.x - per_tensor : blockIdx.x, per_tensor);
  const int bh = id / blocks, b = bh / c.H_kv, in_pair = id - bh * blocks;
  const bool lead = in_pair < range.lead_blocks;
  const Lengths len = lengths_of(c, b);
  const long long first = lead ? 0 : range.first_of != nullptr ? max(range.first_of[b], 0) : window_base(len.total(), range.window);
  const long long block = first / kGroup + in_pair - (lead ? 0 : range.lead_blocks), at = block * kGroup;
  const long long end = min(first + (lead ? range.lead : range.T), (long long)len.total());
  if (at >= end) return;
  const long long row0 = bh * range.pair_rows + (lead ? 0 : range.lead);
  OUT* out = (values ? v_out : k_out) + row0 * kHeadDim;
  const LowTarget low = {range.low.rows + row0 * 4, range.low.scale + row0};
  const int from = (int)max(first, at), to = (int)min(end, at + kGroup);  // positions this workgroup writes
  // with sliding values, the newest 128 tokens' values are the window's: token t in slot t % 128
  const bool sliding = (c.flags & KVLINC_FLAG_SLIDING_VALUES) != 0 && values && len.nq % kGroup == 0;
  const int packed = sliding ? min(len.nq, max(len.total() - kGroup, 0)) : len.nq;
  if (from < packed) {
    const uint32_t* rec = c.groups + ((long long)bh * c.max_groups + block) * Rec<BITS>::kWords;
    const Target<OUT> target = {out, first, from, min(to, packed), (int)at};
    if (values) read_values<BITS, OUT, ROTATED>(rec, all[wave], target, wave, lane);
    else read_keys<BITS, OUT, LOW>(rec, all[wave], target, low, wave, lane);
  }
  const int raw = max(from, packed);
  if (raw >= to) return;
  const int slot0 = sliding ? 0 : len.nq;  // slot of position t: t - nq, or t % 128 where values slide (nq is a multiple of 128 there)
  auto slot_of = [&](int t) { return sliding ? t & (kGroup - 1) : t - slot0; };
  if (!values) {
    const half_t* keys = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
    for (int t = raw + wave; t < to; t += 4) {
      const half2_t k = *reinterpret_cast<const half2_t*>(keys + slot_of(t) * kHeadDim + 2 * lane);
      OUT* dst = out + (t - first) * kHeadDim + 2 * lane;
      dst[0] = rounded<OUT>((float)k[0]);
      dst[1] = rounded<OUT>((float)k[1]);
      if constexpr (LOW) {  // (binary16 numbers as they are)
        if (lane < 16) reinterpret_cast<uint32_t*>(low.rows + (t - first) * 4)[lane] = 0u;
        else if (lane == 16) low.scale[t - first] = 0x7f7f7f7fu;
      }
    }
    return;
  }
  const half_t* vals = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  const int s_first = slot_of(raw), s_last = slot_of(to - 1);  // (a block's slots are consecutive)
  for (int quad = s_first / 4 + wave; quad <= s_last / 4; quad += 4) {
    const uint4 w = reinterpret_cast<const uint4*>(vals + (long long)quad * kHeadDim * 4)[lane];  // channels 2 lane, 2 lane + 1, four slots each
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)as_h2(u[i >> 1])[i & 1];  // [channel][slot]
    if constexpr (!ROTATED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = v[i], d = v[4 + i];
        v[i] = a + d;
        v[4 + i] = a - d;
      }
      lane_butterflies<8>(v, lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= kInvSqrtD;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * quad + i;
      if (slot < s_first || slot > s_last) continue;
      OUT* dst = out + (raw + slot - s_first - first) * kHeadDim + 2 * lane;
      dst[0] = rounded<OUT>(v[i]);
      dst[1] = rounded<OUT>(v[4 + i]);
    }
  }
}

template <int BITS, typename OUT>
int launch_read_of(const kvlinc_cache& c, ReadRange r, void* k_out, void* v_out, bool rotated, hipStream_t stream) {
  // (a range that does not start on a block of 128 touches one more; none has more than the cache)
  const long long of_rows = ((long long)r.T + kGroup - 1) / kGroup, of_cache = c.max_groups + 1;
  const long long blocks = r.lead_blocks + (of_rows < of_cache ? of_rows : of_cache) + (r.first_of != nullptr || r.window > 0 ? 1 : 0);
  const long long per_tensor = blocks * c.B * c.H_kv, grid = per_tensor * ((k_out != nullptr) + (v_out != nullptr));
  if (grid >= (1ll << 24)) return KVLINC_EINVAL;  // 2^32 threads: more than the outputs of any card
  r.blocks = (int)blocks;
  r.per_tensor = (int)per_tensor;
  OUT *k = static_cast<OUT*>(k_out), *v = static_cast<OUT*>(v_out);
  void (*kernel)(kvlinc_cache, ReadRange, OUT*, OUT*) = rotated ? read_kernel<BITS, OUT, true, false> : read_kernel<BITS, OUT, false, false>;
  if constexpr (std::is_same<OUT, half_t>::value)
    if (r.low.rows != nullptr) kernel = read_kernel<BITS, OUT, true, true>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, stream, c, r, k, v);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace

int launch_read(const kvlinc_cache& c, const int32_t* first, int T, void* k_out, void* v_out, int dtype, bool rotated, hipStream_t stream) {
  const ReadRange r = {first, 0, T, 0, 0, T, 0, 0, {nullptr, nullptr}};
  switch (dtype) {
    case KVLINC_F16: return c.bits == 2 ? launch_read_of<2, half_t>(c, r, k_out, v_out, rotated, stream) : launch_read_of<4, half_t>(c, r, k_out, v_out, rotated, stream);
    case KVLINC_BF16: return c.bits == 2 ? launch_read_of<2, BF16>(c, r, k_out, v_out, rotated, stream) : launch_read_of<4, BF16>(c, r, k_out, v_out, rotated, stream);
    default: return c.bits == 2 ? launch_read_of<2, float>(c, r, k_out, v_out, rotated, stream) : launch_read_of<4, float>(c, r, k_out, v_out, rotated, stream);
  }
}

int launch_read_rows(const ContextCall& a, hipStream_t stream) {
  const ReadRange r = {nullptr, a.row_window, a.cached_rows - a.sink_rows, a.sink_rows, (a.sink_rows + kGroup - 1) / kGroup, a.cached_rows, 0, 0,
                       {reinterpret_cast<u32x4_t*>(a.k_low), a.k_low_scale}};
  return a.cache.bits == 2 ? launch_read_of<2, half_t>(a.cache, r, a.k_rows, a.v_rows, true, stream) : launch_read_of<4, half_t>(a.cache, r, a.k_rows, a.v_rows, true, stream);
}

}  // namespace kvlinc
