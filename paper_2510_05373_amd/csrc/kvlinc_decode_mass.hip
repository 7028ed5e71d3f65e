// One decode step that also accumulates what attention weight every group of tokens has received.
//
// The walk over the packed cache is that of kvlinc_rows.hip (shared in kvlinc_row_parts.h) with one token a sequence: a wave takes groups of 128
// packed tokens, or 32 of the window's, and the rows of a KV head, its 1 to 8 query heads, are the columns of the products, each 4 or 2 times for
// different blocks of tokens.  Scores there are exact to about 2^-21 of their terms, which the weights need that are results themselves.
// A weight is known only when the whole context has been seen.  So every wave leaves, for each group and column, its reference and its sum of weights, 128
// bytes a group beside the 9216 or 17408 it reads; and who joins the splits of a pair, and so knows the maximum M and the sum L of every head, makes
//     mass[j] = decay mass[j] + sum over heads of 2^(reference - M) sum / L,
// the columns and heads always in the same order.  No second pass over keys, no second launch.
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_join.h"
#include "kvlinc_row_parts.h"

namespace kvlinc {
namespace {

constexpr int kMaxWaves = 8;

// {reference, sum} of a column: stores and loads past the caches that are not coherent across the chip.
__device__ __forceinline__ void put_sum(unsigned long long* at, float reference, float sum) {
  const unsigned long long v = (unsigned long long)__builtin_bit_cast(uint32_t, sum) << 32 | __builtin_bit_cast(uint32_t, reference);
  __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
struct ColumnSum {
  float reference, sum;
};
__device__ __forceinline__ ColumnSum get_sum(const unsigned long long* at) {
  const unsigned long long v = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  return ColumnSum{__builtin_bit_cast(float, (uint32_t)v), __builtin_bit_cast(float, (uint32_t)(v >> 32))};
}
__device__ __forceinline__ float column_sum(float v) {  // over the four lanes of a column
  float x, y;
  pair_across<16>(v, x, y);
  pair_across<32>(x + y, x, y);
  return x + y;
}

// Grid, one-dimensional: pairs fastest, then the splits.
template <int BITS, int S, bool SLIDING>
__global__ __launch_bounds__(64 * kMaxWaves, 2) void decode_mass_kernel(MassCall a) {
  constexpr int kRows = 16 / S, kAccStride = kHeadDim + 4;
  __shared__ __align__(16) u32x4_t sMeta[kMaxWaves][64];
  __shared__ __align__(16) float sAcc[kMaxWaves][16][kAccStride];
  __shared__ float sM[kMaxWaves][16], sL[kMaxWaves][16];
  __shared__ float sRowM[kRows], sRowL[kRows];
  __shared__ int sLast;
  static_assert(sizeof(sMeta) >= 32 * kMaxContextSplits * sizeof(float), "shared in turn");
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, g = lane >> 4;
  const int pairs = c.B * c.H_kv, split = blockIdx.x / pairs, bh = blockIdx.x - split * pairs;
  const int b = bh / c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int total = len.total(), G = len.groups();
  const long long row0 = (long long)bh * gq;  // (one token a sequence: rows are heads)
  unsigned long long* sums = a.sums + bh * a.slots * 16;
  const bool direct = a.splits == 1;
  const __amdgpu_buffer_rsrc_t part = buffer_of(a.part + (direct ? 0 : row0 * a.splits * kPartStride), direct ? 0 : (long long)gq * a.splits * kPartBytes);

  {
    Rows st;
    st.subset = (lane & 15) / kRows;
    st.m = -INFINITY;
    st.l = st.mid = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) st.acc[n] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto q_row = [&]() __attribute__((always_inline)) { return a.q + (row0 + min(lane & (kRows - 1), gq - 1)) * kHeadDim + 32 * g; };
    load_query(st, q_row(), lane);
    st.p = total - 1;
    st.low = 0;
    const int n_win = (len.nr + kRawTokens - 1) / kRawTokens, step = waves * a.splits;
    int item = split * waves + wave;
    const half_t* k_win = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
    const half_t* v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
    const int quads = c.R / 4;
    for (; item < n_win; item += step) {
      const int t0 = item * kRawTokens;
      float x[2][4];
      raw_weights(st, q_row, k_win + t0 * kHeadDim, len.nq + t0, min(len.nr - t0, kRawTokens), 0, lane, x);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i / 4][i % 4];
      sum = column_sum(sum);
      if (g == 0) put_sum(sums + (long long)(G + item) * 16 + lane, st.m, sum);
      window_values<2>(st, v_win, quads, t0 / 16, x, lane);
    }
    item -= n_win;
    const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
    // (the newest group is left to the code below where its tokens from n_res on take the window's values)
    const int plain = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup && G > 0 ? G - 1 : G;
    if (item < G) {
      Record<BITS> rec;
      load_key_part<BITS>(rec, rec0 + (long long)item * Rec<BITS>::kWords, lane);
      load_value_part<BITS>(rec, rec0 + (long long)item * Rec<BITS>::kWords, lane);
      while (item < plain) {
        const int at = item * kGroup, count = min(len.nq - at, kGroup);
        const bool more = item + step < G;
        const GroupMagnitudes mag = put_meta<BITS>(rec, sMeta[wave], lane);
        float x[8 / S][4], unit, base;
        group_scores<BITS, S>(st, rec, sMeta[wave], mag.key_scale, q_row, at, count, count < kGroup, 0, lane, x, unit, base);
        const uint32_t* next = rec0 + (long long)(more ? item + step : item) * Rec<BITS>::kWords;
        if (more) load_key_part<BITS>(rec, next, lane);
        const float sum = column_sum(group_values<BITS, S, false>(st, rec, sMeta[wave], mag.value_exponent, x, unit, base, kGroup, v_win, quads, lane));
        if (more) load_value_part<BITS>(rec, next, lane);
        if (g == 0) put_sum(sums + (long long)item * 16 + lane, st.m, sum);
        item += step;
      }
      if (SLIDING && item < G) {
        const GroupMagnitudes mag = put_meta<BITS>(rec, sMeta[wave], lane);
        float x[8 / S][4], unit, base;
        group_scores<BITS, S>(st, rec, sMeta[wave], mag.key_scale, q_row, item * kGroup, kGroup, false, 0, lane, x, unit, base);
        const float sum = column_sum(group_values<BITS, S, true>(st, rec, sMeta[wave], mag.value_exponent, x, unit, base, len.nr, v_win, quads, lane));
        if (g == 0) put_sum(sums + (long long)item * 16 + lane, st.m, sum);
      }
    }

    // ---- the waves joined ----
    const float l = column_sum(st.l), mid = column_sum(st.mid);
    if (g == 0) { sM[wave][lane] = reference_of(st.m, l); sL[wave][lane] = l; }
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float4_t v = st.acc[n];
      *reinterpret_cast<float4_t*>(&sAcc[wave][lane & 15][16 * n + 4 * g]) = float4_t{v[0] + mid, v[1] + mid, v[2] + mid, v[3] + mid};
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums are where everybody sees them
  __syncthreads();
  const int r = tid >> 4, ch = 8 * (lane & 15);  // 16 lanes a row
  if (r < gq) {
    float M = -INFINITY;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int u = 0; u < S; ++u) M = fmaxf(M, sM[w][u * kRows + r]);
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, L = 0.0f;
    if (M != -INFINITY) {
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int u = 0; u < S; ++u) {
          const int col = u * kRows + r;
          const float f = __builtin_amdgcn_exp2f(sM[w][col] - M);  // 0 for a column that has seen nothing
          L = fmaf(f, sL[w][col], L);
          const float4_t u0 = *reinterpret_cast<const float4_t*>(&sAcc[w][col][ch]), u1 = *reinterpret_cast<const float4_t*>(&sAcc[w][col][ch + 4]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            o[i] = fmaf(f, u0[i], o[i]);
            o[4 + i] = fmaf(f, u1[i], o[4 + i]);
          }
        }
    }
    if (direct) {
      finish_row(o, L, lane, a.out + (row0 + r) * kHeadDim);
      if ((lane & 15) == 0) { sRowM[r] = M; sRowL[r] = L; }
    } else {
      const int place = (r * a.splits + split) * kPartBytes;
      if ((lane & 15) == 0) store2(part, place, M, L);
      store4(part, place + 16 + 4 * ch, o[0], o[1], o[2], o[3]);
      store4(part, place + 32 + 4 * ch, o[4], o[5], o[6], o[7]);
    }
  }

  // ---- whoever arrives last at the pair's counter joins its splits, and clears the counter ----
  if (!direct) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) sLast = __hip_atomic_fetch_add(c.split_done + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) == a.splits - 1;
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(sLast)) return;
    if (r < gq) {
      float o[8], L, M;
      join_row(part, r * a.splits * kPartBytes, a.splits, reinterpret_cast<float*>(&sMeta[0][0]) + kMaxContextSplits * r, lane, o, L, M);
      finish_row(o, L, lane, a.out + (row0 + r) * kHeadDim);
      if ((lane & 15) == 0) { sRowM[r] = M; sRowL[r] = L; }
    }
    if (tid == 0) c.split_done[bh] = 0;
  }
  __syncthreads();

  // ---- the mass: 16 lanes a slot, a column each ----
  const int col = lane & 15, row = col % kRows;
  const bool used = row < gq;
  const float M = used ? sRowM[row] : 0.0f, L = used ? sRowL[row] : 0.0f;
  const float inv = L != 0.0f ? 1.0f / L : 0.0f;
  const int n_win = (len.nr + kRawTokens - 1) / kRawTokens;
  const long long at = (long long)bh * (c.max_groups + 1);
  for (int j = tid >> 4; j <= G; j += blockDim.x >> 4) {
    const int parts = j < G ? 1 : n_win;
    float w = 0.0f;
    for (int i = 0; i < parts; ++i) {
      const ColumnSum s = get_sum(sums + (long long)(j + i) * 16 + col);
      if (used && s.sum != 0.0f) w = fmaf(s.sum * inv, __builtin_amdgcn_exp2f(s.reference - M), w);
    }
    w += dpp_f<kRowRor1>(w);
    w += dpp_f<kRowRor2>(w);
    w += dpp_f<kRowRor4>(w);
    w += dpp_f<kRowRor8>(w);
    if (col == 0) a.mass_out[at + j] = a.mass != nullptr ? fmaf(a.decay, a.mass[at + j], w) : w;
  }
}

}  // namespace

template <int BITS, int S>
static void launch_of(const MassCall& a, dim3 grid, int waves, hipStream_t stream) {
  if ((a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0) hipLaunchKernelGGL((decode_mass_kernel<BITS, S, true>), grid, dim3(64 * waves), 0, stream, a);
  else hipLaunchKernelGGL((decode_mass_kernel<BITS, S, false>), grid, dim3(64 * waves), 0, stream, a);
}

int launch_decode_mass(const MassCall& a, int waves, hipStream_t stream) {
  const dim3 grid((unsigned)((long long)a.cache.B * a.cache.H_kv * a.splits));
  if (a.cache.bits == 2) a.gq <= 4 ? launch_of<2, 4>(a, grid, waves, stream) : launch_of<2, 2>(a, grid, waves, stream);
  else a.gq <= 4 ? launch_of<4, 4>(a, grid, waves, stream) : launch_of<4, 2>(a, grid, waves, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
