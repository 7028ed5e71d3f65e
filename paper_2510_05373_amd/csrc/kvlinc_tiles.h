// Blocks of 256 query rows over tiles of 64 tokens: what the two kernels of this kind share (not part of the C ABI).  See kvlinc_prompt.hip
// for the layout of rows and products and for the schedule.
#pragma once

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"
#include "kvlinc_reference.h"

namespace kvlinc {
namespace {

constexpr int kTileWaves = 8, kTileThreads = 64 * kTileWaves, kTileRows = 32 * kTileWaves;

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x6_t __attribute__((ext_vector_type(6)));
typedef half_t half32_t __attribute__((ext_vector_type(32)));

// All waves' LDS traffic done, then the next phase; nothing is moved across it.
__device__ __forceinline__ void next_phase() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ---- a wave's rows ----------------------------------------------------------------------------------------------------------------
struct TileRows {
  half8_t q[8];      // channels 16 s + 8 h + 0..7 of this lane's row
  float m, l;        // reference (log2 domain), per-lane sum of the weights
  bool far;          // some row's reference is beyond kFusedBound (the same in all lanes)
  float16_t acc[4];  // numerator of channels 32 cb + 8 (r / 4) + 4 h + r % 4
  float16_t s[2];    // scores of tokens 32 tb + 8 (r / 4) + 4 h + r % 4
  half8_t p[4];      // weights, 16 tokens a step
};

__device__ __forceinline__ void raise_reference(TileRows& st, float largest) {  // largest score of this lane, log2 domain
  if (__builtin_amdgcn_ballot_w64(passes(largest, st.m)) == 0) return;
  float x, y;
  pair_across<32>(largest, x, y);
  const float to = raised(fmaxf(x, y), st.m), f = raised_factor(st.m, to);
  st.m = to;
  st.l *= f;
  st.far = __builtin_amdgcn_ballot_w64(to != -INFINITY && fabsf(to) > kFusedBound) != 0;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) st.acc[cb] *= f;
}

__device__ __forceinline__ half8_t lds_operand(const void* tile, int at) {
  return as_h8(*reinterpret_cast<const u32x4_t*>(static_cast<const char*>(tile) + at));
}
// Order of a matrix phase of MFMAS products: kAhead operands are requested before the first, then one with every product.  (Left to itself
// the compiler keeps two under way, and every pair of products waits for LDS.)
constexpr int kAhead = 6;
template <int MFMAS>
__device__ __forceinline__ void matrix_order() {
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
  for (int i = 0; i < MFMAS - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
}
// ---- what dequantized keys lose --------------------------------------------------------------------------------------------------------
// A key code * scale + zero-point rounded to binary16 is off by up to 2^-12 of itself, and a score by 2^-12 of a sum of |q k|: several times what
// all other roundings of an output come to (8.9e-4 of its norm against 2.5e-4, 512 tokens over 8192 cached ones).  What the rounding leaves is kept as
// FP4 numbers with a scale for every 32 channels, and its products with the query, in FP6, are added to the scores: 2.9e-4 (4 bits 3.4e-4, by the
// rounding of values).  That is 4 products of four times the depth on top of a tile's 32 and a quarter of the keys' bytes: 9 % of a long call, in the kernel
// that unpacks the codes itself, 65 to 512 rows, a quarter.  (A second binary16 term would be 16 products, half of a tile's.)
struct LowTile {
  u32x4_t k[kTileTokens][4];      // 32 channels a chunk; chunk c of token t lies at low_chunk(t, c)
  uint32_t scale[kTileTokens];    // byte c: exponent (biased by 127) of the scale of chunk c
};
__device__ __forceinline__ int low_chunk(int t, int c) { return c ^ ((t >> 2) & 3); }

typedef int i32x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ i32x8_t fp6_operand(u32x6_t v) { return i32x8_t{(int)v[0], (int)v[1], (int)v[2], (int)v[3], (int)v[4], (int)v[5], 0, 0}; }
__device__ __forceinline__ i32x8_t fp4_operand(u32x4_t v) { return i32x8_t{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }
struct LowQuery {
  u32x6_t q[2];  // channels 64 j + 32 h + 0..31 of this lane's row as FP6 (E2M3) numbers
  int scale;     // exponents of their scales in bytes j
};
__device__ __forceinline__ LowQuery low_query(const half_t* q, int lane) {
  LowQuery r;
  r.scale = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const u32x4_t* part = reinterpret_cast<const u32x4_t*>(q + 64 * j + 32 * (lane >> 5));
    u32x4_t x[4];
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      x[c] = part[c];
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(x[c][i] & 0x7fffu, (x[c][i] >> 16) & 0x7fffu));
    }
    const uint32_t e = max(top >> 10, 1u) + 110u;  // the largest is 4 .. 8 of the scale (FP6 ends at 7.5)
    half32_t v;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[8 * c + i] = as_h8(x[c])[i];
    r.q[j] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_f16(v, bits_f32(e << 23));
    r.scale |= (int)(e << (8 * j));
  }
  return r;
}
// v_mfma_scale_f32_32x32x64_f8f6f4: lane l has row l % 32, of the depth 32 (l / 32) .. + 31, under one scale.
__device__ __forceinline__ void low_scores(TileRows& st, const LowTile& t, const LowQuery& q, int lane) {
  const int i = lane & 31, h = lane >> 5;
  int scale[2];
  u32x4_t k[2][2];
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) {
    scale[tb] = (int)(t.scale[32 * tb + i] >> (8 * h));
#pragma unroll
    for (int j = 0; j < 2; ++j) k[tb][j] = t.k[32 * tb + i][low_chunk(i, 2 * j + h)];
  }
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) st.s[tb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(k[tb][0]), fp6_operand(q.q[0]), st.s[tb], 4, 2, 0, scale[tb], 0, q.scale);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) st.s[tb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(k[tb][1]), fp6_operand(q.q[1]), st.s[tb], 4, 2, 2, scale[tb], 1, q.scale);
  __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
  __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
}

// Scores to weights.  masked: not every row sees all tokens of the tile, the first of which is at position `at` (p, low: of this lane's row).
__device__ __forceinline__ void tile_weights(TileRows& st, int at, int count, bool masked, int p, int low, int sinks, int lane) {
  const int h = lane >> 5;
  if (masked) {  // in terms of the token within the tile: seen if t < end and (t >= from or t < first)
    const int end = min(count, p - at + 1) - 4 * h, from = low - at - 4 * h, first = sinks - at - 4 * h;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int t = 32 * tb + 8 * (r >> 2) + (r & 3);
        const bool seen = (t < end) & ((t >= from) | (t < first));
        st.s[tb][r] = seen ? st.s[tb][r] : -INFINITY;
      }
  }
  float mx = st.s[0][0];
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st.s[tb][r]);
  raise_reference(st, mx * kLog2eSqrtD);
  const float m = st.m == -INFINITY ? 0.0f : st.m;
  if (st.far) {
    // The reference was rounded as a product before the head room came off it; so is the score here, or the rounding of the reference
    // itself, thousands up there, would be the exponent of the largest weight.  What is left for the shared code: score - reference.
#pragma clang fp contract(off)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.s[tb][r] = (st.s[tb][r] * kLog2eSqrtD - m) * (1.0f / kLog2eSqrtD);
  }
  const float base = st.far ? 0.0f : -m;
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.s[tb][r] = __builtin_amdgcn_exp2f(fmaf(st.s[tb][r], kLog2eSqrtD, base));
  // (the sum takes the weights as rounded, in binary32: what all of them are rounded by in common cancels in the quotient)
  const half2_t ones = {(half_t)1.0f, (half_t)1.0f};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    half2_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 8 * (k & 1) + 2 * u;
      w[u] = pack_h2(st.s[k >> 1][r], st.s[k >> 1][r + 1]);
      st.l = __builtin_amdgcn_fdot2(w[u], ones, st.l, false);
    }
    st.p[k] = as_h8(w[0], w[1], w[2], w[3]);
  }
}

// acc H, in binary32.
__device__ __forceinline__ void rotate_tile_rows(TileRows& st, int lane) {
  const float s32 = (lane & 32) != 0 ? -1.0f : 1.0f;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) {
#pragma unroll
    for (int hb = 1; hb < 16; hb *= 2)  // channel bits 0, 1 (r % 4) and 3, 4 (r / 4)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if ((r & hb) == 0) {
          const float a = st.acc[cb][r], b = st.acc[cb][r + hb];
          st.acc[cb][r] = a + b;
          st.acc[cb][r + hb] = a - b;
        }
#pragma unroll
    for (int r = 0; r < 16; ++r) {  // bit 2: the halves of the wave
      float x, y;
      pair_across<32>(st.acc[cb][r], x, y);
      st.acc[cb][r] = __builtin_fmaf(y, s32, x) * kInvSqrtD;
    }
  }
#pragma unroll
  for (int hb = 1; hb < 4; hb *= 2)
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
      if ((cb & hb) == 0) {
        const float16_t a = st.acc[cb], b = st.acc[cb + hb];
        st.acc[cb] = a + b;
        st.acc[cb + hb] = a - b;
      }
}

// Work items of the grid: split fastest, then (sequence, KV head), blocks of rows from the last (the longest) to the first.  Workgroups are
// dealt to the 8 XCDs in turn: where the pairs divide by 8, those of one pair are 8 apart, so that its tiles come from one L2.  Within an XCD they
// are dealt to its 4 shader engines in turn, too, and wait for theirs: the pairs change places from block to block, or four long sequences
// among short ones would be one engine's work each (4 prompts of 1700 to 4096 rows: some compute units idle for 473 of 548 us).
struct BlockPlace {
  int split, bh, block;
};
__device__ __forceinline__ BlockPlace place_of_block(const ContextCall& a, int blocks) {
  const int pairs = a.cache.B * a.cache.H_kv, id = blockIdx.x;
  BlockPlace p;
  if (pairs % 8 == 0) {
    const int x = id & 7, y = id >> 3, per = pairs / 8, rest = y / a.splits;
    p.split = y - rest * a.splits;
    p.block = rest / per;
    p.bh = (rest - p.block * per + p.block) % per * 8 + x;
  } else {
    const int rest = id / a.splits;
    p.split = id - rest * a.splits;
    p.block = rest / pairs;
    p.bh = rest - p.block * pairs;
  }
  p.block = blocks - 1 - p.block;
  return p;
}

// A row that sees one of the tokens of a tile whose values are not finite (`bad`, a bit each; in the tile they are zeros) becomes not a number.
__device__ __forceinline__ uint64_t bits_below(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }
__device__ __forceinline__ void spoil_rows(TileRows& st, uint64_t bad, int at, int p, int low, int sinks) {
  const uint64_t seen = bits_below(p - at + 1) & (~bits_below(low - at) | bits_below(sinks - at));
  if ((seen & bad) != 0) st.l = NAN;
}

// The rows of a wave.
struct WaveRows {
  bool idle, mine;          // no row of the wave, or this lane's, is one of the call's (lanes beyond the last row take it along)
  long long place;          // of this lane's row
  int p, low;               // its position, the first token of its window
  int p_first, p_last;      // positions of the wave's first and last row
  int low_first, low_last;  // and the first tokens of their windows
};
__device__ __forceinline__ WaveRows wave_rows(const ContextCall& a, int b, int kvh, int rows, int first, int total, int lane) {
  WaveRows w;
  const int row = min(first + (lane & 31), rows - 1), i = row / a.gq, h = row - i * a.gq;
  w.idle = first >= rows;
  w.mine = first + (lane & 31) < rows;
  w.place = ((long long)b * a.cache.H_q + (long long)kvh * a.gq + h) * a.T + i;
  w.p = total + i;
  w.low = window_low(w.p, a.window);
  w.p_first = __builtin_amdgcn_readfirstlane(total + min(first, rows - 1) / a.gq);
  w.p_last = __builtin_amdgcn_readfirstlane(total + min(first + 31, rows - 1) / a.gq);
  w.low_first = window_low(w.p_first, a.window);
  w.low_last = window_low(w.p_last, a.window);
  return w;
}
// Whether some row of the wave sees a token of a tile, and whether some row does not see all 64.
__device__ __forceinline__ bool wave_sees(const WaveRows& w, const ContextCall& a, int at, int count) {
  return !w.idle && at <= w.p_last && (at + count > w.low_first || at < a.sinks);
}
__device__ __forceinline__ bool wave_masked(const WaveRows& w, const ContextCall& a, int at, int count) {
  return count < kTileTokens || at + kTileTokens - 1 > w.p_first || (at < w.low_last && at + kTileTokens > a.sinks);
}

__device__ __forceinline__ void start_rows(TileRows& st, const half_t* q, int lane) {
  const uint4* src = reinterpret_cast<const uint4*>(q) + (lane >> 5);
#pragma unroll
  for (int k = 0; k < 8; ++k) st.q[k] = as_h8(src[2 * k]);
  st.m = -INFINITY;
  st.l = 0.0f;
  st.far = false;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.acc[cb][r] = 0.0f;
}

// What the block leaves: a split's partial result, or the output row -- with the correction, normalised, in the original basis.
__device__ __forceinline__ void store_results(TileRows& st, const ContextCall& a, const WaveRows& w, int split, bool in_cache_basis, int lane) {
  if (w.idle) return;
  const int h = lane >> 5;
  {
    float x, y;
    pair_across<32>(st.l, x, y);
    st.l = x + y;
  }
  if (a.splits > 1) {
    if (!w.mine) return;
    float* dst = a.part + (w.place * a.splits + split) * kPartStride;
    if (h == 0) { dst[0] = reference_of(st.m, st.l); dst[1] = st.l; }
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(dst + 4 + 32 * cb + 2 * r + 4 * h) = make_float4(st.acc[cb][r], st.acc[cb][r + 1], st.acc[cb][r + 2], st.acc[cb][r + 3]);
    return;
  }
  if (a.corr != nullptr) {  // {C_d, -, -, -, C_n[128]}
    const float* corr = a.corr + w.place * kPartStride;
    const Shares f = shares_of(st.m, corr[0]);
    st.l = fmaf(f.correction, corr[0], st.l * f.softmax);
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 v = *reinterpret_cast<const float4*>(corr + 4 + 32 * cb + 2 * r + 4 * h);
        st.acc[cb][r] = fmaf(f.correction, v.x, st.acc[cb][r] * f.softmax);
        st.acc[cb][r + 1] = fmaf(f.correction, v.y, st.acc[cb][r + 1] * f.softmax);
        st.acc[cb][r + 2] = fmaf(f.correction, v.z, st.acc[cb][r + 2] * f.softmax);
        st.acc[cb][r + 3] = fmaf(f.correction, v.w, st.acc[cb][r + 3] * f.softmax);
      }
  }
  if (in_cache_basis) rotate_tile_rows(st, lane);
  if (!w.mine) return;
  const float inv = 1.0f / st.l;
  half_t* dst = a.out + w.place * kHeadDim;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<uint2*>(dst + 32 * cb + 2 * r + 4 * h) =
          make_uint2(as_u32(pack_h2(st.acc[cb][r] * inv, st.acc[cb][r + 1] * inv)), as_u32(pack_h2(st.acc[cb][r + 2] * inv, st.acc[cb][r + 3] * inv)));
}

}  // namespace
}  // namespace kvlinc
