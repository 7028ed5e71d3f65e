// What query rows add to the accumulated attention weight of the groups, without their output rows.
//
// Three steps.  scores_kernel leaves, for every row and slot (a group, or the window), log2 of the row's sum of weights over the slot's tokens;
// rows_kernel makes of them the same over all tokens that the row sees; and columns_kernel sums 2^(the first - the second) over the rows of a slot.
// So the weights are formed once, groups do not wait for one another, and what goes through memory is 4 bytes a row and group.  Where a pair's numbers fit into
// LDS one workgroup takes the last two steps (masses_of_pair), in a launch of its own or in the first one.
// Bound: matrix work with vector work beside it, see below: 2048 rows of 8 pairs of 4 heads over 32768 tokens 790 us (two products: 1.4 PFLOP/s), of which the
// last two steps take 27; 32 rows of 128 pairs over up to 8192 tokens 69 us, the longest sequence's 4 groups a wave and 8 blocks of rows (1.75 us each; launch,
// the rows' way to LDS, first record, arrival and the last two steps the rest, some 16).  At 4 bits 874 and 76: keys take more to unpack, and <4, false> and
// <4, true> spill 5 and 10 registers.  Waves of a workgroup share slots, not blocks of rows: where a sequence has fewer slots than four, some have nothing to do.
// 64 prompts with all of their rows, 8 pairs of 4 heads each: of 100 tokens 56 us (a copy of the rows 11), 250 157 (27), 500 398 (54); one of 8192 511 (one
// product 227).
//
// scores_kernel.  S^T = K Q^T on v_mfma_f32_16x16x32_f16: codes as binary16 numbers, query times key scales in two binary16 terms (exactness as in
// kvlinc_rows.hip).  A wave unpacks a group's key tile into 128 registers and goes over blocks of 16 rows with it: 64 products, 32 exponentials a lane.
// Zero-points and centring are two sums over channels, products of rows, too.  Vector work goes ahead of products (s_setprio): the two waves of a
// SIMD, with the same steps to do, otherwise do them side by side, products then vector work, and neither fills the other's gaps (2048 rows over 32768
// tokens: 887 us, 810 so).  The second term as FP6 numbers, half of the matrix work, was 793 (its conversion takes 20 issue slots) and 30 times less
// exact; four FP6 terms and codes as they lie 1085.
// A column's reference is one that an earlier group has left, as long as the sums it gives stay below 2^14; only where they do not, the largest score is
// looked for and the weights are formed again: what a row's larger weights leave of a slot below 2^-126 of them is nothing.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_join.h"
#include "kvlinc_row_parts.h"

namespace kvlinc {
namespace {

constexpr int kScoreWaves = 4, kMostBlocks = 8;           // blocks of 16 rows of a workgroup
constexpr int kQueryStride = kHeadDim + 8;                // halves of a row in LDS
constexpr float kMostSum = 0x1p14f;

// Rows and tokens of a sequence.
struct Place {
  Lengths len;
  int rows, T;  // rows of a KV head, rows of a query head
  bool beyond;  // more tokens than the caller's bound: no rows
  __device__ __forceinline__ int position(int row, int gq) const { return len.total() - T + row / gq; }
};
__device__ __forceinline__ Place place_of(const MassCall& a, int b) {
  const Lengths len = lengths_of(a.cache, b);
  const int T = a.n_rows != nullptr ? min(max(a.n_rows[b], 0), a.T) : a.T;
  const bool beyond = len.total() > a.bound;
  return Place{len, beyond ? 0 : T * a.gq, T, beyond};
}

template <int BITS>
struct KeyPart {
  u32x4_t kw[2 * BITS];
  u32x4_t meta;  // lanes 0..31: scales, zero-points
};
template <int BITS>
__device__ __forceinline__ void load_keys_of(KeyPart<BITS>& r, const uint32_t* rec, int lane) {
  const u32x4_t* kt = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyTile) + token_order(lane & 15) + (lane & 48);
#pragma unroll
  for (int m = 0; m < 2 * BITS; ++m) r.kw[m] = kt[64 * m];
  r.meta = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyScale)[lane & 31];
}

// Scores of a tile of 128 tokens become a column's sum of weights relative to col.m (-inf: nothing seen yet), which may be raised.
struct Column {
  float m;
};
__device__ __forceinline__ float tile_sum(Column& col, float4_t (&x)[8], float unit, float bias) {
  float4_t l4 = {0.f, 0.f, 0.f, 0.f};
  const float base = bias - col.m;
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) l4[r] += __builtin_amdgcn_exp2f(fmaf(x[n][r], unit, base));
  float l = (l4[0] + l4[1]) + (l4[2] + l4[3]);
  if (__builtin_amdgcn_ballot_w64(!(l <= kMostSum) || fmaxf(fabsf(bias), fabsf(col.m)) > kFusedBound) != 0) {
    float mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[n][r] = fmaf(x[n][r], unit, bias);
        mx = fmaxf(mx, x[n][r]);
      }
    float a, b;
    pair_across<16>(mx, a, b);
    pair_across<32>(fmaxf(a, b), a, b);
    col.m = raised(fmaxf(a, b), col.m);
    const float m = finite_reference(col.m);
    l = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) l += __builtin_amdgcn_exp2f(x[n][r] - m);
  }
  float a, b;
  pair_across<16>(l, a, b);
  pair_across<32>(a + b, a, b);
  return a + b;
}
// Tokens 16 n + pi(4 g + r) from `end` on are not seen.
__device__ __forceinline__ void hide_from(float4_t (&x)[8], int end, int g) {
#pragma unroll
  for (int n = 0; n < 8; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) x[n][r] = 16 * n + token_order(4 * g + r) >= end ? -INFINITY : x[n][r];
}

// The mass of a pair from log2 of its rows' sums, by a workgroup: the numbers in LDS, [slots][rows], the sums of the rows over their slots, a thread four
// rows and a part of the slots, and those of the slots over their rows, 16 threads a slot.  COHERENT: other workgroups of the launch have left them.
template <int THREADS, bool COHERENT>
__device__ __forceinline__ void masses_of_pair(const MassCall& a, const Place& at, int bh, float* sLse, float* sRow /* LDS, 4 THREADS */) {
  const int tid = threadIdx.x, G = at.len.groups(), rows = a.rows;
  // unlike scores_kernel's, numbers of slots that a row does not see are read here, and left
  const auto first_of = [&](int slot) { return slot < G ? slot * kGroup : at.len.nq; };
  float* lse = a.lse + (long long)bh * a.slots * rows;
  const int slots = at.rows == 0 ? 0 : G + (at.len.nr > 0 ? 1 : 0);
  const __amdgpu_buffer_rsrc_t from_others = buffer_of(lse, COHERENT ? slots * rows * 4 : 0);
#pragma unroll 8
  for (int i = 4 * tid; i < slots * rows; i += 4 * THREADS)
    *reinterpret_cast<float4_t*>(sLse + i) = COHERENT ? load4(from_others, 4 * i) : *reinterpret_cast<const float4_t*>(lse + i);
  __syncthreads();
  const int quads = rows / 4, parts = min(THREADS / quads, slots), quad = tid % quads, part = tid / quads;
  if (part < parts) {
    int p[4];
    float m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] = at.position(min(4 * quad + i, at.rows - 1), a.gq);
      m[i] = -INFINITY;
      l[i] = 0.0f;
    }
#pragma unroll 4
    for (int s = part; s < slots; s += parts) {
      const float4_t v = *reinterpret_cast<const float4_t*>(sLse + s * rows + 4 * quad);
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = fmaxf(m[i], first_of(s) <= p[i] ? v[i] : -INFINITY);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = finite_reference(m[i]);
#pragma unroll 4
    for (int s = part; s < slots; s += parts) {
      const float4_t v = *reinterpret_cast<const float4_t*>(sLse + s * rows + 4 * quad);
#pragma unroll
      for (int i = 0; i < 4; ++i) l[i] += __builtin_amdgcn_exp2f(first_of(s) <= p[i] ? v[i] - m[i] : -INFINITY);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sRow[part * rows + 4 * quad + i] = m[i] + __builtin_amdgcn_logf(l[i]);  // (-inf: it sees none of them)
  }
  __syncthreads();
  for (int row = tid; row < rows && slots > 0; row += THREADS) {
    float M = -INFINITY, L = 0.0f;
    for (int i = 0; i < parts; ++i) M = fmaxf(M, sRow[i * rows + row]);
    M = finite_reference(M);
    for (int i = 0; i < parts; ++i) L += __builtin_amdgcn_exp2f(sRow[i * rows + row] - M);
    sRow[row] = M + __builtin_amdgcn_logf(L);  // (nobody else reads this row's)
  }
  __syncthreads();
  const int of_slot = tid & 15;
  for (int slot = tid >> 4; slot <= G; slot += THREADS / 16) {
    const int from = max(first_of(slot) - (at.len.total() - at.T), 0) * a.gq;  // rows before that of the first token do not see it
    float w = 0.0f;
    for (int r = 4 * of_slot; slot < slots && r < at.rows; r += 64) {
      const float4_t v = *reinterpret_cast<const float4_t*>(sLse + slot * rows + r), to = *reinterpret_cast<const float4_t*>(sRow + r);
#pragma unroll
      for (int i = 0; i < 4; ++i) w += __builtin_amdgcn_exp2f(r + i >= from && r + i < at.rows ? v[i] - to[i] : -INFINITY);
    }
    w += dpp_f<kRowRor1>(w);
    w += dpp_f<kRowRor2>(w);
    w += dpp_f<kRowRor4>(w);
    w += dpp_f<kRowRor8>(w);
    const long long column = (long long)bh * (a.cache.max_groups + 1) + slot;
    if (of_slot == 0) a.mass_out[column] = a.mass != nullptr ? fmaf(a.decay, a.mass[column], w) : w;
  }
  if (at.beyond && bh % a.cache.H_kv == 0 && tid == 0) atomicOr(a.cache.status, KVLINC_ST_BOUND);
}

// Grid, one-dimensional: pairs fastest, then runs of kScoreWaves splits of the slots, then sets of a.blocks blocks of rows.
// WHOLE: a pair's numbers, kWholeNumbers at most of kWholeRows, fit into the LDS that the queries leave: its workgroup that arrives last at the pair's
// counter (zero before and after) forms the mass of them.
constexpr int kWholeNumbers = kMostBlocks * 16 * kQueryStride / 2, kWholeRows = 64 * kScoreWaves;
template <int BITS, bool WHOLE>
__global__ __launch_bounds__(64 * kScoreWaves, 2) void scores_kernel(MassCall a, int blocks, int runs) {
  __shared__ __align__(16) float sNumbers[kWholeNumbers];
  half_t (*sQuery)[kQueryStride] = reinterpret_cast<half_t (*)[kQueryStride]>(sNumbers);
  __shared__ __align__(16) float sRow[WHOLE ? 4 * 64 * kScoreWaves : 1];
  __shared__ __align__(16) u32x4_t sMeta[kScoreWaves][33];  // key scales, zero-points, zeros
  __shared__ float sUnit[kMostBlocks * 16], sRef[kScoreWaves][kMostBlocks * 16];
  __shared__ int sPosition[kMostBlocks * 16], sLossy;
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, g = lane >> 4;
  const int pairs = c.B * c.H_kv, unit_id = blockIdx.x / pairs, bh = blockIdx.x - unit_id * pairs, set = unit_id / runs, split = (unit_id - set * runs) * kScoreWaves + wave;
  const int b = bh / c.H_kv, gq = a.gq, row0 = 16 * blocks * set;
  const Place at = place_of(a, b);
  if (row0 >= at.rows) {
    if constexpr (WHOLE) {
      if (at.rows == 0 && unit_id == 0) masses_of_pair<64 * kScoreWaves, true>(a, at, bh, sNumbers, sRow);
    }
    return;
  }
  const int G = at.len.groups(), splits = runs * kScoreWaves, n_blocks = min(blocks, (at.rows - row0 + 15) / 16);
  if (!WHOLE && at.position(min(row0 + 16 * n_blocks, at.rows) - 1, gq) < 0) return;  // (rows ahead of the first token)
  const long long head0 = (long long)bh * gq;
  auto query_of = [&](int row) {  // (rows beyond the last take its query)
    const RowPlace p = row_place(min(row, at.rows - 1), gq);
    return a.q + ((head0 + p.h) * a.T + p.i) * kHeadDim;
  };

  // ---- the rows to LDS, as load_query of kvlinc_row_parts.h has them ----
  if (tid == 0) sLossy = 0;
  __syncthreads();
  for (int row = tid >> 4; row < 16 * n_blocks; row += 4 * kScoreWaves) {
    const u32x4_t raw = reinterpret_cast<const u32x4_t*>(query_of(row0 + row))[lane & 15];
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = max(mx, max(raw[i] & 0x7fffu, (raw[i] >> 16) & 0x7fffu));
    mx = max(mx, dpp_u<kRowRor1>(mx));
    mx = max(mx, dpp_u<kRowRor2>(mx));
    mx = max(mx, dpp_u<kRowRor4>(mx));
    mx = max(mx, dpp_u<kRowRor8>(mx));
    const QueryScale by = query_scale(mx);
    u32x4_t scaled;
    uint32_t lost = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      scaled[i] = as_u32(as_h2(raw[i]) * by.by);
      lost |= as_u32(as_h2(scaled[i]) * by.back) ^ raw[i];
    }
    *reinterpret_cast<u32x4_t*>(&sQuery[row][8 * (lane & 15)]) = scaled;
    if (lost != 0) sLossy = 1;
    if ((lane & 15) == 0) {
      sUnit[row] = by.unit;
      sPosition[row] = at.position(min(row0 + row, at.rows - 1), gq);
    }
  }
  for (int k = 0; k < n_blocks; ++k) sRef[wave][16 * k + j] = -INFINITY;
  if (lane == 0) sMeta[wave][32] = u32x4_t{0, 0, 0, 0};
  __syncthreads();

  float* lse = a.lse + bh * a.slots * a.rows + row0;
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
  const bool lossy = __builtin_amdgcn_readfirstlane(sLossy) != 0;
  const int oldest = __builtin_amdgcn_readfirstlane(sPosition[0]), newest = __builtin_amdgcn_readfirstlane(sPosition[16 * n_blocks - 1]);
  auto load_rows = [&](int k, half8_t (&q)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const half8_t*>(&sQuery[16 * k + j][32 * g + 8 * s]);
  };
  auto leave = [&](int slot, int k, const Column& col, float sum) __attribute__((always_inline)) {
    sRef[wave][16 * k + j] = col.m;  // (the same in the four lanes of a column: each reads what it has written)
    if (g != 0) return;
    float* to = lse + (long long)slot * a.rows + 16 * k + j;
    const float of_slot = finite_reference(col.m) + __builtin_amdgcn_logf(sum);
    if constexpr (WHOLE) __hip_atomic_store(to, of_slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    else *to = of_slot;
  };
  // What the zero-points and the centring add to a score is a product, too: of rows that are the zero-points (in every quarter's first row of the
  // product) and the scales (in the second), so that every lane finds both sums of its column.
  const int bias_at = (j & 3) == 0 ? 16 + 4 * g : (j & 3) == 1 ? 4 * g : 32, bias_step = (j & 3) < 2 ? 1 : 0;
  KeyPart<BITS> rec;
  int slot = split;
  if (slot < G) load_keys_of<BITS>(rec, rec0 + (long long)slot * Rec<BITS>::kWords, lane);
  for (; slot < G && slot * kGroup <= newest; slot += splits) {
    const int first = slot * kGroup, count = min(at.len.nq - first, kGroup);
    if (lane < 32) sMeta[wave][lane] = rec.meta;
    wave_order();
    // scales are not negative: their bit patterns order like the numbers
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(rec.meta[i] & 0xffffu, rec.meta[i] >> 16));
    top = max(top, dpp_u<kRowRor1>(top));
    top = max(top, dpp_u<kRowRor2>(top));
    top = max(top, dpp_u<kRowRor4>(top));
    top = max(top, dpp_u<kRowRor8>(top));
    const bool wide = lossy || (uint32_t)__builtin_amdgcn_readlane(top, 0) >= kFirstLargeScale;  // (lanes 0..15 have the scales)
    const bool masked = count < kGroup || first + kGroup - 1 > oldest;
    half8_t A[8][4];
#pragma unroll
    for (int n = 0; n < 8; ++n) key_operands<BITS>(rec.kw, n, A[n]);
    const int next = slot + splits < G ? slot + splits : slot;
    load_keys_of<BITS>(rec, rec0 + (long long)next * Rec<BITS>::kWords, lane);
    auto block = [&](int k, auto general) __attribute__((always_inline)) {
      constexpr bool kGeneral = decltype(general)::value;
      float bias, unit = sUnit[16 * k + j];
      Column col = {sRef[wave][16 * k + j]};
      half8_t hi[4], lo[4];
      if (kGeneral && wide) {
        wide_operands<BITS>(query_of(row0 + 16 * k + j) + 32 * g, &sMeta[wave][0], lane, hi, lo, bias, unit);
      } else {
        half8_t q[4];
        load_rows(k, q);
        float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(sMeta[wave][bias_at + s * bias_step]), q[s], d, 0, 0, 0);
          const u32x4_t sc = sMeta[wave][4 * g + s], qq = __builtin_bit_cast(u32x4_t, q[s]);
          u32x4_t h, r;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const half2_t x = as_h2(qq[i]), y = as_h2(sc[i]), t = x * y;
            h[i] = as_u32(t);
            r[i] = as_u32(__builtin_elementwise_fma(x, y, -t));
          }
          hi[s] = as_h8(h);
          lo[s] = as_h8(r);
        }
        bias = fmaf(d[1], Rec<BITS>::kCentre, d[0]) * unit;
      }
      __builtin_amdgcn_s_setprio(0);
      float4_t x[8];
#pragma unroll
      for (int n = 0; n < 8; ++n) x[n] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[n][s], lo[s], x[n], 0, 0, 0);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[n][s], hi[s], x[n], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      if (kGeneral && masked) hide_from(x, min(count, sPosition[16 * k + j] - first + 1), g);
      const float sum = tile_sum(col, x, unit, bias);
      leave(slot, k, col, sum);
    };
    if (wide || masked) {
      for (int k = 0; k < n_blocks; ++k)  // (a block of rows goes over a slot whose first token its last row sees)
        if (first <= __builtin_amdgcn_readfirstlane(sPosition[16 * k + 15])) block(k, std::true_type{});
    } else {
      for (int k = 0; k < n_blocks; ++k) block(k, std::false_type{});
    }
    wave_order();
  }
  // ---- the window's raw rows, by the wave whose turn it is ----
  if (at.len.nr > 0 && G % splits == split && at.len.nq <= newest) {
    const half_t* keys = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
    half8_t A[8][4];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const u32x4_t* row = reinterpret_cast<const u32x4_t*>(keys + (long long)min(16 * n + token_order(j), at.len.nr - 1) * kHeadDim + 32 * g);
#pragma unroll
      for (int s = 0; s < 4; ++s) A[n][s] = as_h8(row[s]);
    }
    for (int k = 0; k < n_blocks; ++k) {
      if (at.len.nq > __builtin_amdgcn_readfirstlane(sPosition[16 * k + 15])) continue;
      half8_t q[4];
      float unit = sUnit[16 * k + j];
      load_rows(k, q);
      if (lossy) {
        const u32x4_t* src = reinterpret_cast<const u32x4_t*>(query_of(row0 + 16 * k + j) + 32 * g);
#pragma unroll
        for (int s = 0; s < 4; ++s) q[s] = as_h8(src[s]);
        unit = kLog2eSqrtD;
      }
      float4_t x[8];
#pragma unroll
      for (int n = 0; n < 8; ++n) x[n] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int n = 0; n < 8; ++n) x[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[n][s], q[s], x[n], 0, 0, 0);
      hide_from(x, min(at.len.nr, sPosition[16 * k + j] - at.len.nq + 1), g);
      Column col = {sRef[wave][16 * k + j]};
      const float sum = tile_sum(col, x, unit, 0.0f);
      leave(G, k, col, sum);
    }
  }
  if constexpr (WHOLE) {
    const int workgroups = (at.rows + 16 * blocks - 1) / (16 * blocks) * runs;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's numbers are where everybody sees them
    __syncthreads();
    if (tid == 0) sLossy = __hip_atomic_fetch_add(c.split_done + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) == workgroups - 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(sLossy) == 0) return;
    if (tid == 0) c.split_done[bh] = 0;
    masses_of_pair<64 * kScoreWaves, true>(a, at, bh, sNumbers, sRow);
  }
}

// Slots whose first token a row at position p sees: groups 0 .. n - 1, and the window.
struct Seen {
  int groups;
  bool window;
};
__device__ __forceinline__ Seen seen_by(const Lengths& len, int p) { return Seen{p < 0 ? 0 : min(p / kGroup + 1, len.groups()), len.nr > 0 && p >= len.nq}; }

// log2 of a row's sum over all it sees.  Grid: pairs by runs of 64 rows, pairs fastest; a lane a row, the slots shared by the waves.
constexpr int kRowWaves = 16;
__global__ __launch_bounds__(64 * kRowWaves) void rows_kernel(MassCall a) {
  __shared__ float sM[kRowWaves][64], sL[kRowWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.cache.B * a.cache.H_kv, run = blockIdx.x / pairs, bh = blockIdx.x - run * pairs;
  const int row = 64 * run + lane;
  const Place at = place_of(a, bh / a.cache.H_kv);
  if (64 * run >= at.rows || at.position(min(64 * run + 63, at.rows - 1), a.gq) < 0) return;
  const Seen see = seen_by(at.len, row < at.rows ? at.position(row, a.gq) : -1);
  const int G = at.len.groups(), slots = see.groups;
  const float* lse = a.lse + bh * a.slots * a.rows + min(row, at.rows - 1);
  // two passes, the second from the caches: the largest first
  constexpr int kAhead = 8;
  float m = -INFINITY;
  for (int s0 = wave; s0 < slots; s0 += kAhead * kRowWaves) {
    float v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = lse[(long long)min(s0 + i * kRowWaves, slots - 1) * a.rows];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) m = fmaxf(m, v[i]);
  }
  const bool window = wave == 0 && see.window;
  const float of_window = window ? lse[(long long)G * a.rows] : -INFINITY;
  m = finite_reference(fmaxf(m, of_window));
  float l = window ? __builtin_amdgcn_exp2f(of_window - m) : 0.0f;
  for (int s0 = wave; s0 < slots; s0 += kAhead * kRowWaves) {
    float v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = lse[(long long)min(s0 + i * kRowWaves, slots - 1) * a.rows];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) l += s0 + i * kRowWaves < slots ? __builtin_amdgcn_exp2f(v[i] - m) : 0.0f;
  }
  sM[wave][lane] = l == 0.0f ? -INFINITY : m;
  sL[wave][lane] = l;
  __syncthreads();
  if (wave != 0 || row >= at.rows) return;
  float M = -INFINITY, L = 0.0f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) M = fmaxf(M, sM[w][lane]);
  const float to = finite_reference(M);
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) L = fmaf(__builtin_amdgcn_exp2f(sM[w][lane] - to), sL[w][lane], L);
  a.row_lse[(long long)bh * a.rows + row] = to + __builtin_amdgcn_logf(L);
}

// Both of what follows scores_kernel in one launch, a workgroup a pair, where its numbers fit into LDS.
constexpr int kPairThreads = 1024, kPairNumbers = 32768;
__global__ __launch_bounds__(kPairThreads) void pair_kernel(MassCall a) {
  extern __shared__ __align__(16) float sLse[];  // [slots][rows]
  __shared__ __align__(16) float sRow[4 * kPairThreads];
  const Place at = place_of(a, blockIdx.x / a.cache.H_kv);
  masses_of_pair<kPairThreads, false>(a, at, blockIdx.x, sLse, sRow);
}

// The mass.  Grid: a wave a slot, those of a pair one after the other.
constexpr int kColumnWaves = 4;
__global__ __launch_bounds__(64 * kColumnWaves) void columns_kernel(MassCall a, long long columns) {
  const int lane = threadIdx.x & 63;
  const long long column = (long long)blockIdx.x * kColumnWaves + (threadIdx.x >> 6);
  if (column >= columns) return;
  const long long bh = column / (a.cache.max_groups + 1);
  const int slot = (int)(column - bh * (a.cache.max_groups + 1)), b = (int)(bh / a.cache.H_kv);
  const Place at = place_of(a, b);
  const int G = at.len.groups();
  if (slot > G) return;
  if (slot == G && at.beyond && bh % a.cache.H_kv == 0 && lane == 0) atomicOr(a.cache.status, KVLINC_ST_BOUND);
  const int first = slot < G ? slot * kGroup : at.len.nq;  // rows before that of the first token do not see it
  const int from = at.rows == 0 ? 0 : max(first - (at.len.total() - at.T), 0) * a.gq;
  const float* lse = a.lse + (bh * a.slots + slot) * a.rows;
  const float* of_row = a.row_lse + bh * a.rows;
  float w = 0.0f;
  if (slot < G || at.len.nr > 0) {
    const auto add = [&](int row) __attribute__((always_inline)) {  // (rows of a pair begin at 64 bytes)
      const float4_t v = *reinterpret_cast<const float4_t*>(lse + row), l = *reinterpret_cast<const float4_t*>(of_row + row);
#pragma unroll
      for (int i = 0; i < 4; ++i) w += row + i >= from && row + i < at.rows ? __builtin_amdgcn_exp2f(v[i] - l[i]) : 0.0f;
    };
    int row = (from & ~255) + 4 * lane;
    for (; row + 3 * 256 < at.rows; row += 4 * 256) {
#pragma unroll
      for (int u = 0; u < 4; ++u) add(row + 256 * u);
    }
    for (; row < at.rows; row += 256) add(row);
  }
  w = wave_allsum(w);
  if (lane == 0) a.mass_out[column] = a.mass != nullptr ? fmaf(a.decay, a.mass[column], w) : w;
}

}  // namespace

int launch_attention_mass(const MassCall& a, hipStream_t stream) {
  const long long pairs = (long long)a.cache.B * a.cache.H_kv, row_blocks = a.rows / 16;
  // Some 2048 waves, two a SIMD; blocks of rows share an unpacked tile where there are more of them and of groups than that.
  long long blocks = pairs * row_blocks * a.slots / 2048;
  blocks = blocks < 1 ? 1 : blocks > kMostBlocks ? kMostBlocks : blocks;
  if (blocks > row_blocks) blocks = row_blocks;
  const long long sets = (row_blocks + blocks - 1) / blocks;
  long long splits = 2048 / (pairs * sets);
  if (splits > a.slots) splits = a.slots;
  if (splits < 1) splits = 1;
  const long long runs = (splits + kScoreWaves - 1) / kScoreWaves;
  const dim3 grid((unsigned)(pairs * sets * runs)), block(64 * kScoreWaves);
  // One launch with few numbers (8 pairs of 128 rows: 700 tokens 8.6 us for 11.2) or many pairs (64 sequences of 2048 tokens 71 us for 76.6); few pairs of many
  // numbers have more threads in a launch of their own (one sequence of 4096 tokens 13.1 us for 15.2).
  const bool whole = a.rows <= kWholeRows && a.slots * a.rows <= (pairs < 32 ? kWholeNumbers / 4 : kWholeNumbers);
  void (*scores)(MassCall, int, int) = a.cache.bits == 2 ? (whole ? scores_kernel<2, true> : scores_kernel<2, false>) : (whole ? scores_kernel<4, true> : scores_kernel<4, false>);
  hipLaunchKernelGGL(scores, grid, block, 0, stream, a, (int)blocks, (int)runs);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  if (whole) return KVLINC_OK;
  if (a.rows <= kPairThreads && a.slots * a.rows <= kPairNumbers) {
    hipLaunchKernelGGL(pair_kernel, dim3((unsigned)pairs), dim3(kPairThreads), (size_t)(a.slots * a.rows) * sizeof(float), stream, a);
    return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
  }
  hipLaunchKernelGGL(rows_kernel, dim3((unsigned)(pairs * ((a.rows + 63) / 64))), dim3(64 * kRowWaves), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  const long long columns = pairs * (a.cache.max_groups + 1);
  hipLaunchKernelGGL(columns_kernel, dim3((unsigned)((columns + kColumnWaves - 1) / kColumnWaves)), dim3(64 * kColumnWaves), 0, stream, a, columns);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
