// Prompt attention of few query rows (up to 64 of a KV head), read directly from the packed cache.
//
// One launch.  Rows of a (sequence, KV head) are (token i, head h) pairs, row = i gq + h.  A workgroup has all rows of one and a split of its
// tokens; a wave takes a block of 16 rows and blocks of tokens on its own, without a barrier: groups of 128 packed tokens, or 32 raw ones (the
// cache's window, the new rows), and keeps a running maximum, sum and numerator.  The waves are joined through LDS, the splits and the
// correction (a workgroup of its own, ahead of the others in the grid) through memory, by whoever arrives last at the counter of the pair.
//
// Both products run on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T (rows = tokens, columns = query rows) and
// O^T = V^T P^T (rows = channels, columns = query rows), so that a lane holds one query row, lane % 16, throughout, and the weights it
// forms are the operand it feeds.  For that the tokens of a block of 16 are taken in the order pi(4 g + r) = 8 (g % 2) + 2 (g / 2) +
// r % 2 + 4 (r / 2) (g = lane / 16): what a lane of the second product has of a value tile's words.
// Codes become binary16 numbers code - centre in one instruction a pair and stay unscaled: the key scales ride on the query (q s in two binary16
// terms, the second what the first leaves: together 2^-22 of q s, or 2^-31 of the row's largest |q|, whichever is more), the value scales on the weights.
// With the scale on the tile instead, every group would cost 128 multiply-adds a lane and 16 rows, where this takes 32; the second term keeps the scores
// as exact as binary32 products of the scales would be.  Magnitudes that binary16 has no room for take the same products the long way (wide_operands).
// Zero-points and centring are sums over channels resp. tokens.
// Bound: vector instructions, some 740 a wave, 16 rows and group of 128 tokens (beside 96 products), two waves a SIMD; and for few pairs the join of
// their splits, two trips to memory past the caches, 7 to 9 us.  16 sequences of 8k tokens, 8 KV heads of 4: 1 token 27 us, 4 tokens 28.5 (3.0 TB/s), with
// the correction 30.5, 4 bits 41; one of 131072: 6 tokens (24 rows, two blocks that both unpack the codes), correction, 51 us.
// Weights are rounded to binary16 once, for the second product: 2^-12 of each at most, of no common sign.  They are kept near 2^8 (see
// kvlinc_reference.h), where the smallest that count are normal numbers; sums of weights are taken before the rounding, in binary32.
#include <hip/hip_runtime.h>

#include "kvlinc_codes.h"
#include "kvlinc_features.h"
#include "kvlinc_join.h"
#include "kvlinc_row_parts.h"

namespace kvlinc {
namespace {

constexpr int kMaxWaves = 8;

// O^T += V^T P^T with raw value rows of 128 halves.  A lane gathers the 8 values of a channel (16 lanes: 32 contiguous bytes a row).  A row that
// sees a value that is not finite becomes not a number; the others take it as 0.
__device__ __forceinline__ void raw_values(Rows& st, const half_t* values, int count, const float (&w)[2][4], uint32_t seen_bits, int lane) {
  const int g = lane >> 4;
  const half8_t P = as_h8(pack_h2(w[0][0], w[0][1]), pack_h2(w[0][2], w[0][3]), pack_h2(w[1][0], w[1][1]), pack_h2(w[1][2], w[1][3]));
  const half_t* row[8];
#pragma unroll
  for (int u = 0; u < 8; ++u)
    row[u] = values + (long long)min(16 * (u >> 2) + token_order(4 * g + (u & 3)), count - 1) * kHeadDim + (lane & 15);
  u32x4_t V[8];
  uint32_t bad = 0;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    half8_t v;
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = row[u][16 * n];
    V[n] = __builtin_bit_cast(u32x4_t, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= not_finite(V[n][i]);
  }
  if (__builtin_amdgcn_ballot_w64(bad != 0) != 0) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {  // (the 16 lanes of g have the channels of the same tokens)
      uint32_t of_token = 0;
#pragma unroll
      for (int n = 0; n < 8; ++n) of_token |= not_finite(V[n][u >> 1]) >> (15 + 16 * (u & 1)) & 1u;
      const uint64_t lanes = __builtin_amdgcn_ballot_w64(of_token != 0);
      if ((lanes >> (16 * g) & 0xffffu) != 0 && (seen_bits >> u & 1u) != 0) st.l = NAN;
    }
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) V[n][i] = finite_or_zero(V[n][i]);
  }
#pragma unroll
  for (int n = 0; n < 8; ++n) st.acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(V[n]), P, st.acc[n], 0, 0, 0);
}

// acc H: channels 16 n + 4 g + r, seven butterfly stages and the factor 1 / sqrt(128), in binary32.
__device__ __forceinline__ void rotate_rows(Rows& st, int lane) {
  const float s16 = (lane & 16) != 0 ? -1.0f : 1.0f, s32 = (lane & 32) != 0 ? -1.0f : 1.0f;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float4_t v = st.acc[n];
    const float a0 = v[0] + v[1], a1 = v[0] - v[1], a2 = v[2] + v[3], a3 = v[2] - v[3];
    float t[4] = {a0 + a2, a1 + a3, a0 - a2, a1 - a3};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x, y;
      pair_across<16>(t[r], x, y);
      t[r] = __builtin_fmaf(y, s16, x);
      pair_across<32>(t[r], x, y);
      st.acc[n][r] = __builtin_fmaf(y, s32, x) * kInvSqrtD;
    }
  }
#pragma unroll
  for (int h = 1; h < 8; h *= 2)
#pragma unroll
    for (int n = 0; n < 8; ++n)
      if ((n & h) == 0) {
        const float4_t a = st.acc[n], b = st.acc[n + h];
        st.acc[n] = a + b;
        st.acc[n + h] = a - b;
      }
}

// ---- the correction of all rows of a pair (Sec. 3.2, Eq. 5-6), by one workgroup ----------------------------------------------------------------
// Products: kvlinc_features.h.  First the features, a wave a head and half of them at a time (16 tokens as columns), through LDS;
// then C_n^T = S^T phi^T, a wave a block of 16 channels, so that the state is read once for all heads.
constexpr int kFeatureStride = kRank + 8;  // halves of a row in LDS
__device__ __forceinline__ void correct_rows(const ContextCall& a, int b, int kvh, int T, int rows, int wave, int waves, int lane, half_t* features, float (*den)[64]) {
  const kvlinc_cache& c = a.cache;
  const int j = lane & 15, g = lane >> 4, gq = a.gq;
  const long long kv = (long long)b * c.H_kv + kvh, head0 = (long long)b * c.H_q + (long long)kvh * gq;
  for (int unit = wave; unit < 2 * gq; unit += waves) {
    const int h = unit >> 1, half = unit & 1;
    const half_t* W = reinterpret_cast<const half_t*>(c.Wq) + (((long long)kvh * gq + h) * 2 + half) * kHeadDim * 128;
    const float* P = c.P + kv * kRank + 128 * half;
    for (int i0 = 0; i0 < T; i0 += 16) {
      const u32x4_t* src = reinterpret_cast<const u32x4_t*>(a.q + ((head0 + h) * a.T + min(i0 + j, T - 1)) * kHeadDim) + g;
      half8_t q[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) q[s] = as_h8(src[4 * s]);  // channels 32 s + 8 g + 0..7
      float4_t d[2][4];  // [64-feature block][tile]: features 64 fb + 16 g + 4 r + i
#pragma unroll
      for (int fb = 0; fb < 2; ++fb) {
#pragma unroll
        for (int i = 0; i < 4; ++i) d[fb][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          u32x4_t w[4];
          weight_operands(W, s, fb, j, g, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) d[fb][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(w[i]), q[s], d[fb][i], 0, 0, 0);
        }
        asm volatile("" ::: "memory");  // (the loads of both blocks at once would spill)
      }
      half8_t phi[2][2];
      const float p = column_features(d, P, g, phi);
      const int row = (i0 + j) * gq + h;
      if (i0 + j < T) {
        if (g == 0) den[half][row] = p;
#pragma unroll
        for (int fb = 0; fb < 2; ++fb)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            *reinterpret_cast<half8_t*>(features + row * kFeatureStride + 128 * half + 64 * fb + 16 * g + 8 * e) = phi[fb][e];
      }
    }
  }
  __syncthreads();
  const half_t* S = reinterpret_cast<const half_t*>(c.S16) + kv * (128 * 64 * 4);
  const __amdgpu_buffer_rsrc_t out = buffer_of(a.corr + head0 * a.T * kPartStride, (long long)gq * a.T * kPartBytes);
  for (int n = wave; n < 8; n += waves) {
    half8_t A[8];  // features 32 s + 8 g + 0..7 of channel 16 n + j
#pragma unroll
    for (int s = 0; s < 8; ++s) A[s] = as_h8(state_operand(S, 32 * s + 8 * g, 16 * n + j));
    for (int r0 = 0; r0 < rows; r0 += 16) {
      const int row = r0 + j;
      float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 8; ++s)
        d = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[s], *reinterpret_cast<const half8_t*>(features + min(row, rows - 1) * kFeatureStride + 32 * s + 8 * g), d, 0, 0, 0);
      if (row < rows) {
        const RowPlace at = row_place(row, gq);
        const int place = (at.h * a.T + at.i) * kPartBytes;
        if (n == 0 && g == 0) store2(out, place, den[0][row] + den[1][row], 0.0f);
        store4(out, place + 16 + 64 * n + 16 * g, d[0], d[1], d[2], d[3]);
      }
    }
  }
}

// Grid, one-dimensional: with the correction, one workgroup a (sequence, KV head) for it; then the splits, pairs fastest.  Up to 64 rows a pair.
template <int BITS, int S, bool SLIDING>
__global__ __launch_bounds__(64 * kMaxWaves, 2) void rows_kernel(ContextCall a) {
  constexpr int kBlockRows = 16 / S, kAccStride = kHeadDim + 4;
  __shared__ __align__(16) u32x4_t sMeta[kMaxWaves][64];
  __shared__ __align__(16) float sAcc[kMaxWaves][16][kAccStride];
  __shared__ float sM[kMaxWaves][16], sL[kMaxWaves][16];
  __shared__ int sLast;
  static_assert(sizeof(sAcc) >= 64 * kFeatureStride * sizeof(half_t) && sizeof(sMeta) >= 32 * kMaxContextSplits * sizeof(float) && sizeof(sM) + sizeof(sL) >= 2 * 64 * sizeof(float), "shared in turn");
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, g = lane >> 4;
  const int pairs = c.B * c.H_kv, n_corr = a.corr != nullptr ? pairs : 0;
  const bool correction = (int)blockIdx.x < n_corr;
  const int unit = correction ? blockIdx.x : blockIdx.x - n_corr, split = correction ? 0 : unit / pairs, bh = unit - split * pairs;
  const int b = bh / c.H_kv, kvh = bh - b * c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int T = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T;
  const int rows = T * gq;
  if (rows == 0) return;  // (nobody arrives for such a sequence)
  const long long head0 = (long long)b * c.H_q + (long long)kvh * gq;
  const int total = len.total();
  // blocks of rows that the waves share: 1, 2 or 4, whatever this sequence's number of rows
  const int all_blocks = (a.T * gq + kBlockRows - 1) / kBlockRows, blocks = all_blocks <= 2 ? all_blocks : 4;
  const bool direct = a.splits == 1 && a.corr == nullptr;
  const __amdgpu_buffer_rsrc_t part = buffer_of(a.part + (direct ? 0 : head0 * a.T * a.splits * kPartStride), direct ? 0 : (long long)gq * a.T * a.splits * kPartBytes);

  if (correction) {
    correct_rows(a, b, kvh, T, rows, wave, waves, lane, reinterpret_cast<half_t*>(&sAcc[0][0][0]), reinterpret_cast<float (*)[64]>(&sM[0][0]));
  } else {
    const int block = wave % blocks, walker = wave / blocks, walkers = waves / blocks;
    const int row0 = block * kBlockRows;
    Rows st;
    st.subset = S == 1 ? 0 : (lane & 15) / kBlockRows;
    st.m = -INFINITY;
    st.l = st.mid = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) st.acc[n] = float4_t{0.f, 0.f, 0.f, 0.f};
    if (row0 < rows) {
      auto q_row = [&]() __attribute__((always_inline)) {
        const RowPlace at = row_place(min(row0 + (lane & (kBlockRows - 1)), rows - 1), gq);
        return a.q + ((head0 + at.h) * a.T + at.i) * kHeadDim + 32 * g;
      };
      {
        const int i = row_place(min(row0 + (lane & (kBlockRows - 1)), rows - 1), gq).i;
        st.p = total + i;
        st.low = window_low(st.p, a.window);
        load_query(st, q_row(), lane);
      }
      // Blocks of tokens that some row sees: the new rows' (32 each), the window's (32 each), the groups.  `low` is that of the first row, the
      // last row's position ends the new ones.
      const int first_i = row0 / gq, last_i = min(row0 + kBlockRows - 1, rows - 1) / gq;
      const int low = window_low(total + first_i, a.window), low_last = window_low(total + last_i, a.window);
      const int new_from = a.sinks > total ? 0 : max(low - total, 0) / kRawTokens;
      const int n_new = (last_i + kRawTokens) / kRawTokens - new_from;
      const int win_from = a.sinks > len.nq ? 0 : min(max(low - len.nq, 0), len.nr) / kRawTokens;
      const int n_win = (len.nr + kRawTokens - 1) / kRawTokens - win_from;
      const int G = len.groups(), group_low = min(low / kGroup, G);
      const int n_sink = a.window > 0 ? min((int)(((long long)a.sinks + kGroup - 1) / kGroup), group_low) : 0;
      const int n_groups = G - group_low + n_sink;
      const int step = walkers * a.splits;
      int item = split * walkers + walker;

      {
        bool rotate = false;
        const half_t* keys = a.k_new + (long long)bh * a.T * kHeadDim;
        const half_t* values = a.v_new + (long long)bh * a.T * kHeadDim;
        for (; item < n_new; item += step) {
          const int t0 = (new_from + item) * kRawTokens;
          float x[2][4];
          const uint32_t seen_bits = raw_weights(st, q_row, keys + (long long)t0 * kHeadDim, total + t0, min(T - t0, kRawTokens), a.sinks, lane, x);
          raw_values(st, values + (long long)t0 * kHeadDim, min(T - t0, kRawTokens), x, seen_bits, lane);
          rotate = true;
        }
        if (rotate) rotate_rows(st, lane);  // from here on the accumulators are in the cache's rotated basis
      }
      item -= n_new;
      const half_t* k_win = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
      const half_t* v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
      const int quads = c.R / 4;
      for (; item < n_win; item += step) {
        const int t0 = (win_from + item) * kRawTokens;
        float x[2][4];
        raw_weights(st, q_row, k_win + t0 * kHeadDim, len.nq + t0, min(len.nr - t0, kRawTokens), a.sinks, lane, x);
        window_values<2>(st, v_win, quads, t0 / 16, x, lane);
      }
      item -= n_win;
      const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
      auto group_of = [&](int it) { return it < n_sink ? it : it - n_sink + group_low; };
      // (the newest group, the last item, is left to the code below where its tokens from n_res on take the window's values: in the loop that
      // code's registers spilled, and drafts over 16 sequences of 8k tokens took 41 us, 4 bits 71)
      const int plain = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup && n_groups > 0 && group_of(n_groups - 1) == G - 1 ? n_groups - 1 : n_groups;
      if (item < n_groups) {
        Record<BITS> rec;
        int gr = group_of(item);
        load_key_part<BITS>(rec, rec0 + (long long)gr * Rec<BITS>::kWords, lane);
        load_value_part<BITS>(rec, rec0 + (long long)gr * Rec<BITS>::kWords, lane);
        while (item < plain) {
          const int at = gr * kGroup, count = min(len.nq - at, kGroup);
          const bool masked = count < kGroup || (at < low_last && at + kGroup > a.sinks), more = item + step < n_groups;
          const GroupMagnitudes mag = put_meta<BITS>(rec, sMeta[wave], lane);
          float x[8 / S][4], unit, exponent_base;
          group_scores<BITS, S>(st, rec, sMeta[wave], mag.key_scale, q_row, at, count, masked, a.sinks, lane, x, unit, exponent_base);
          const int next = more ? group_of(item + step) : gr;
          if (more) load_key_part<BITS>(rec, rec0 + (long long)next * Rec<BITS>::kWords, lane);
          group_values<BITS, S, false>(st, rec, sMeta[wave], mag.value_exponent, x, unit, exponent_base, kGroup, v_win, quads, lane);
          if (more) load_value_part<BITS>(rec, rec0 + (long long)next * Rec<BITS>::kWords, lane);
          item += step;
          gr = next;
        }
        if (SLIDING && item < n_groups) {
          const int at = gr * kGroup;
          const GroupMagnitudes mag = put_meta<BITS>(rec, sMeta[wave], lane);
          float x[8 / S][4], unit, exponent_base;
          group_scores<BITS, S>(st, rec, sMeta[wave], mag.key_scale, q_row, at, kGroup, at < low_last && at + kGroup > a.sinks, a.sinks, lane, x, unit, exponent_base);
          group_values<BITS, S, true>(st, rec, sMeta[wave], mag.value_exponent, x, unit, exponent_base, len.nr, v_win, quads, lane);
        }
      }
    }

    // ---- the waves joined ----
    {
      float x, y;
      pair_across<16>(st.l, x, y);
      pair_across<32>(x + y, x, y);
      const float l = x + y;
      pair_across<16>(st.mid, x, y);
      pair_across<32>(x + y, x, y);
      const float mid = x + y;
      if (g == 0) { sM[wave][lane] = reference_of(st.m, l); sL[wave][lane] = l; }
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const float4_t v = st.acc[n];
        *reinterpret_cast<float4_t*>(&sAcc[wave][lane & 15][16 * n + 4 * g]) = float4_t{v[0] + mid, v[1] + mid, v[2] + mid, v[3] + mid};
      }
    }
    __syncthreads();
    const int ch = 8 * (lane & 15);
    for (int slot = tid >> 4; slot < blocks * kBlockRows; slot += blockDim.x >> 4) {
      const int blk = slot / kBlockRows, r = slot % kBlockRows, row = slot;
      if (row >= rows) continue;  // (the 16 lanes of a row go together)
      float M = -INFINITY;
      for (int w = blk; w < waves; w += blocks)
#pragma unroll
        for (int u = 0; u < S; ++u) M = fmaxf(M, sM[w][u * kBlockRows + r]);
      float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, L = 0.0f;
      if (M != -INFINITY) {
        for (int w = blk; w < waves; w += blocks)
#pragma unroll
          for (int u = 0; u < S; ++u) {
            const int col = u * kBlockRows + r;
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
      const RowPlace at = row_place(row, gq);
      if (direct) {
        finish_row(o, L, lane, a.out + ((head0 + at.h) * a.T + at.i) * kHeadDim);
      } else {
        const int place = ((at.h * a.T + at.i) * a.splits + split) * kPartBytes;
        if ((lane & 15) == 0) store2(part, place, M, L);
        store4(part, place + 16 + 4 * ch, o[0], o[1], o[2], o[3]);
        store4(part, place + 32 + 4 * ch, o[4], o[5], o[6], o[7]);
      }
    }
    if (direct) return;
  }

  // ---- whoever arrives last at the pair's counter joins its splits and the correction, and clears the counter ----
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's results are where everybody sees them
  __syncthreads();
  if (tid == 0) sLast = __hip_atomic_fetch_add(c.split_done + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) == a.splits - 1 + (a.corr != nullptr ? 1 : 0);
  __syncthreads();
  if (!__builtin_amdgcn_readfirstlane(sLast)) return;
  const __amdgpu_buffer_rsrc_t corr = buffer_of(a.corr + (a.corr != nullptr ? head0 * a.T * kPartStride : 0), a.corr != nullptr ? (long long)gq * a.T * kPartBytes : 0);
  float* weights = reinterpret_cast<float*>(&sMeta[0][0]) + kMaxContextSplits * (tid >> 4);
  for (int row = tid >> 4; row < rows; row += blockDim.x >> 4) {
    const RowPlace at = row_place(row, gq);
    const int place = at.h * a.T + at.i, ch = 8 * (lane & 15);
    float c_d = 0.0f;
    float4_t c0 = {0.f, 0.f, 0.f, 0.f}, c1 = c0;
    if (a.corr != nullptr) {
      c_d = load2(corr, place * kPartBytes)[0];
      c0 = load4(corr, place * kPartBytes + 16 + 4 * ch);
      c1 = load4(corr, place * kPartBytes + 32 + 4 * ch);
    }
    float o[8], L, M;
    join_row(part, place * a.splits * kPartBytes, a.splits, weights, lane, o, L, M);
    if (a.corr != nullptr) add_correction(o, L, M, c_d, c0, c1);
    finish_row(o, L, lane, a.out + ((head0 + at.h) * a.T + at.i) * kHeadDim);
  }
  if (tid == 0) c.split_done[bh] = 0;
}

// The splits of a launch over blocks of 256 rows joined, 16 rows a workgroup.  Row = (b H_q + h) T + i.
__global__ __launch_bounds__(256) void join_kernel(ContextCall a, long long n_rows) {
  const int lane = threadIdx.x & 63, ch = 8 * (lane & 15);
  const long long place = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (place >= n_rows) return;
  if (a.n_new != nullptr) {
    const long long h = place / a.T;
    if (place - h * a.T >= a.n_new[h / a.cache.H_q]) return;
  }
  const float* p = a.part + place * a.splits * kPartStride;
  float M = -INFINITY;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, p[s * kPartStride]);
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, L = 0.0f;
  if (M != -INFINITY)
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      const float* src = p + s * kPartStride;
      const float f = __builtin_amdgcn_exp2f(src[0] - M);
      L = fmaf(f, src[1], L);
      const float4_t u0 = *reinterpret_cast<const float4_t*>(src + 4 + ch), u1 = *reinterpret_cast<const float4_t*>(src + 8 + ch);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i] = fmaf(f, u0[i], o[i]);
        o[4 + i] = fmaf(f, u1[i], o[4 + i]);
      }
    }
  if (a.corr != nullptr) {
    const float* corr = a.corr + place * kPartStride;
    add_correction(o, L, M, corr[0], *reinterpret_cast<const float4_t*>(corr + 4 + ch), *reinterpret_cast<const float4_t*>(corr + 8 + ch));
  }
  finish_row(o, L, lane, a.out + place * kHeadDim);
}

}  // namespace

template <int BITS, int S>
static void launch_rows_of(const ContextCall& a, dim3 grid, int waves, hipStream_t stream) {
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  if (sliding) hipLaunchKernelGGL((rows_kernel<BITS, S, true>), grid, dim3(64 * waves), 0, stream, a);
  else hipLaunchKernelGGL((rows_kernel<BITS, S, false>), grid, dim3(64 * waves), 0, stream, a);
}

int launch_rows(const ContextCall& a, int waves, hipStream_t stream) {
  const int rows = a.T * a.gq;
  const dim3 grid((unsigned)((long long)a.cache.B * a.cache.H_kv * (a.splits + (a.corr != nullptr ? 1 : 0))));
  if (a.cache.bits == 2) rows <= 4 ? launch_rows_of<2, 4>(a, grid, waves, stream) : rows <= 8 ? launch_rows_of<2, 2>(a, grid, waves, stream) : launch_rows_of<2, 1>(a, grid, waves, stream);
  else rows <= 4 ? launch_rows_of<4, 4>(a, grid, waves, stream) : rows <= 8 ? launch_rows_of<4, 2>(a, grid, waves, stream) : launch_rows_of<4, 1>(a, grid, waves, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

int launch_join(const ContextCall& a, hipStream_t stream) {
  const long long n = (long long)a.cache.B * a.cache.H_q * a.T;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)((n + 15) / 16)), dim3(256), 0, stream, a, n);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
