// One decode step that also accumulates what attention weight every group of tokens has received.
//
// The walk over the packed cache is that of kvlinc_windowed.hip without a window (shared in kvlinc_decode_parts.h): codes go to the matrix cores as
// FP4, weights as three FP8 terms, zero-points exact, all query heads of a KV head share one pass.  Weights are results here, so query times key scale
// has four terms (2^-16 of each product, see qk_phase), in the row of the matrix instruction that is spare.
// A weight is known only when the whole context has been seen.  So every wave leaves, for each group and head, its reference and its sum of weights, 64
// bytes a group beside the 9216 or 17408 it reads; and who joins the splits of a pair, and so knows the maximum M and the sum L of every head, makes
//     mass[j] = decay mass[j] + sum over heads of 2^(reference - M) sum / L,
// always in the same order.  No second pass over keys, no second launch.
// Bound: bytes of the groups.  32 sequences of 32k tokens, 7 heads, 4 bits: 119.0 us, 4.9 TB/s; with half of the tokens missing from the shortest 106.5
// (the splits are made for the longest); 16 of 8k, 2 bits: 22.3 us, 3.6 TB/s, of which the chain of counters, first record, arrival, join and mass takes
// 6; one of 300 tokens: 8.4 us, the host's calls.  (The walk of few-row attention, which unpacks the codes for binary16 products: 119.5 for the 106.5,
// 28 for the 22.3.  Two workgroups a compute unit, 512 in all; with 1024 110 and 26, three a unit at 2 bits spill.)
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_decode_parts.h"
#include "kvlinc_join.h"

namespace kvlinc {
namespace {

constexpr int kHalfMirror = 0x141;  // row_half_mirror: lane 7 - i of every 8
constexpr int kSumHeads = 8;    // pairs {reference, sum} of a slot
constexpr int kShare = 32;     // tokens of the window a wave takes, with a slot of their own
constexpr int kSlotsAhead = 8;  // slots of a lane requested together

// {reference, sum} of a head: a store past the caches that are not coherent across the chip.
__device__ __forceinline__ void put_sum(unsigned long long* at, float reference, float sum) { st_coherent2(reinterpret_cast<float*>(at), reference, sum); }

// Grid, one-dimensional: (sequence, KV head) fastest, then the split.
template <int NB, bool SLIDING, int BITS>
__global__ __launch_bounds__(kThreads, 2) void decode_mass_kernel(MassCall a) {
  constexpr int kCombine = 2 * kWaves * NB * 4 + kWaves * NB * 4 * kHeadDim, kRecordWords = Rec<BITS>::kWords, kTerms = 4;
  __shared__ __align__(16) float lds[kCombine + kWaves * 2 * kExWords];
  uint32_t (*ex)[2 * kExWords] = reinterpret_cast<uint32_t (*)[2 * kExWords]>(lds + kCombine);
  __shared__ float sRowM[kSumHeads], sRowL[kSumHeads];
  __shared__ int sLast;
  static_assert(kWaves * 2 * kExWords >= kThreads / 16 * kMaxContextSplits, "weights of the join");
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pairs = c.B * c.H_kv, split = blockIdx.x / pairs, bh = blockIdx.x - split * pairs, b = bh / c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int G = len.groups();
  // every workgroup of the pair comes to the same number: a split has a group for each wave
  const int n_splits = max(1, min(a.splits, (G + kWaves - 1) / kWaves));
  if (split >= n_splits) return;
  const long long row0 = (long long)bh * gq;  // (one token a sequence: rows are heads)
  unsigned long long* const sums = a.sums + bh * a.slots * kSumHeads;

  const Roles lr = make_roles(lane, ex[wave]);
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * kRecordWords;
  GroupOrder order(n_splits, split, wave, BITS == 2 && n_splits > 1 ? 2 : 1);
  int rd = split == 0 ? order.skip : 0, idx = order.group(rd);
  KeyRegs<BITS> kr;
  ValueRegs<BITS> vr;
  if (idx < G) {
    const uint32_t* src = rec0 + (long long)idx * kRecordWords;
    load_keys(kr, src, lr);
    load_values(vr, src, lr);
  }
  uint32_t qh[NB][4];  // q of the head this lane builds operands for (head 4 nb + ha, or the last one), channels c0 .. c0 + 7
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const uint4 raw = *reinterpret_cast<const uint4*>(a.q + (row0 + min(nb * 4 + lr.ha, gq - 1)) * kHeadDim + lr.c0);
    qh[nb][0] = raw.x; qh[nb][1] = raw.y; qh[nb][2] = raw.z; qh[nb][3] = raw.w;
  }
  // the spare term row of the weights' exchange regions reads as zero
#pragma unroll
  for (int k = 0; k < 4; ++k) ex[wave][(k >> 1) * kExWords + (2 * (k & 1) + (lane >> 5)) * kExHead + 96 + (lane & 31)] = 0u;
  lds_order();
  WaveState<NB> st;
  empty_state<NB>(st);
  const auto leave = [&](int slot, const float (&sum)[NB]) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float s = row_allsum(sum[nb]);
      if (lr.jd == 0) put_sum(sums + (long long)slot * kSumHeads + nb * 4 + lr.hd, st.m[nb], s);
    }
  };
  if (split == 0) {
    const WindowShare sh = {kShare * wave, min(kShare * wave + kShare, len.nr)};
    if (sh.first < sh.end) {
      WindowRegs w;
      request_window(w, c, bh, sh, lr);
      window_part<NB>(w, qh, sh, lr, st);
      leave(G + wave, st.l);
    }
  }
  const half_t* const v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  float (*sM)[NB * 4] = reinterpret_cast<float (*)[NB * 4]>(lds);
  float (*sL)[NB * 4] = reinterpret_cast<float (*)[NB * 4]>(lds + kWaves * NB * 4);
  float (*sAcc)[NB * 4][kHeadDim] = reinterpret_cast<float (*)[NB * 4][kHeadDim]>(lds + 2 * kWaves * NB * 4);
  // (the newest group is left to the code below where its tokens from n_res on take the window's values)
  const int plain = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup && G > 0 ? G - 1 : G;
  while (idx < plain) {
    const int next = order.group(++rd);
    const bool more = next < G;
    const uint32_t* src = rec0 + (long long)(more ? next : idx) * kRecordWords;
    float sc[NB][8], off[NB], base[NB], sum[NB];
    qk_phase<NB, BITS, true, kTerms>(kr, min(kGroup, len.nq - idx * kGroup), qh, lr, sc, off);
    if (more) load_keys(kr, src, lr);
    update_reference<NB>(sc, off, base, st, kSlack);
    pv_phase<NB, BITS, false, kTerms>(vr, sc, base, lr, st, kGroup, sum);
    if (more) load_values(vr, src, lr);
    leave(idx, sum);
    idx = next;
  }
  if (SLIDING && idx < G) {
    float sc[NB][8], off[NB], base[NB], sum[NB];
    qk_phase<NB, BITS, true, kTerms>(kr, kGroup, qh, lr, sc, off);
    update_reference<NB>(sc, off, base, st, kSlack);
    pv_phase<NB, BITS, true, kTerms>(vr, sc, base, lr, st, len.nr, sum);
    leave(idx, sum);
    pv_window_tail<NB>(v_win, sc, base, len.nr, lr, st, lane, sAcc[wave]);
  }

  // ---- the waves joined; one (m, l, numerators) a head ----
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float l = row_allsum(st.l[nb]), pz = row_allsum(st.pz[nb]);
    const int h = nb * 4 + lr.hd;
    if (lr.jd == 0) { sM[wave][h] = reference_of(st.m[nb], l); sL[wave][h] = l; }
#pragma unroll
    for (int n = 0; n < 8; ++n) sAcc[wave][h][16 * n + lr.jd] = st.acc[nb][n] + pz;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums are where everybody sees them
  __syncthreads();
  const bool direct = n_splits == 1;
  const __amdgpu_buffer_rsrc_t part = buffer_of(a.part + (direct ? 0 : row0 * a.splits * kPartStride), direct ? 0 : (long long)gq * a.splits * kPartBytes);
  const int h = tid >> 4, ch = 8 * (lane & 15);  // 16 lanes a head
  if (h < gq) {
    float M = -INFINITY, L = 0.0f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sM[w][h]);
    if (M != -INFINITY) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sM[w][h] - M);  // 0 for a wave without tokens
        L = fmaf(f, sL[w][h], L);
        const float4_t u0 = *reinterpret_cast<const float4_t*>(&sAcc[w][h][ch]), u1 = *reinterpret_cast<const float4_t*>(&sAcc[w][h][ch + 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[i] = fmaf(f, u0[i], o[i]);
          o[4 + i] = fmaf(f, u1[i], o[4 + i]);
        }
      }
    }
    if (direct) {
      finish_row(o, L, lane, a.out + (row0 + h) * kHeadDim);
      if ((lane & 15) == 0) { sRowM[h] = M; sRowL[h] = L; }
    } else {
      const int place = (h * a.splits + split) * kPartBytes;
      if ((lane & 15) == 0) store2(part, place, M, L);
      store4(part, place + 16 + 4 * ch, o[0], o[1], o[2], o[3]);
      store4(part, place + 32 + 4 * ch, o[4], o[5], o[6], o[7]);
    }
  }

  // ---- whoever arrives last at the pair's counter joins its splits, and clears the counter ----
  if (!direct) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) sLast = __hip_atomic_fetch_add(c.split_done + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) == n_splits - 1;
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(sLast)) return;
  }

  // ---- the mass: 8 lanes a slot, a head each, kSlotsAhead slots under way, the first of them requested together with the splits' results ----
  const int head = tid & (kSumHeads - 1), n_win = (len.nr + kShare - 1) / kShare, entries = G + n_win;
  const long long at = (long long)bh * (c.max_groups + 1);
  float2 s[kSlotsAhead];
  float before[kSlotsAhead];
  const auto request = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kSlotsAhead; ++i) {
      const int j = j0 + i * (kThreads / kSumHeads);
      s[i] = make_float2(0.0f, 0.0f);
      before[i] = 0.0f;
      if (j < entries && head < NB * 4) s[i] = ld_coherent2(reinterpret_cast<const float*>(sums + (long long)j * kSumHeads + head));
      if (j < G && a.mass != nullptr) before[i] = a.mass[at + j];
    }
  };
  request(tid / kSumHeads);
  if (!direct) {
    if (h < gq) {
      float o[8], L, M;
      join_row(part, h * a.splits * kPartBytes, n_splits, reinterpret_cast<float*>(&ex[0][0]) + kMaxContextSplits * h, lane, o, L, M);
      finish_row(o, L, lane, a.out + (row0 + h) * kHeadDim);
      if ((lane & 15) == 0) { sRowM[h] = M; sRowL[h] = L; }
    }
    if (tid == 0) c.split_done[bh] = 0;
  }
  __syncthreads();
  const bool used = head < gq;
  const float M = used ? sRowM[head] : 0.0f, L = used ? sRowL[head] : 0.0f;
  const float inv = L != 0.0f ? 1.0f / L : 0.0f;
  const auto weight_of = [&](float2 v) __attribute__((always_inline)) {
    float w = used && v.y != 0.0f ? v.y * inv * __builtin_amdgcn_exp2f(v.x - M) : 0.0f;
    w += dpp_f<kQuadSwap1>(w);
    w += dpp_f<kQuadSwap2>(w);
    return w + dpp_f<kHalfMirror>(w);
  };
  float* const sWindow = lds;  // (the combine buffer is read no more)
  for (int j0 = tid / kSumHeads;; request(j0)) {
#pragma unroll
    for (int i = 0; i < kSlotsAhead; ++i) {
      const int j = j0 + i * (kThreads / kSumHeads);
      const float w = weight_of(s[i]);
      if (head != 0 || j >= entries) continue;
      if (j < G) a.mass_out[at + j] = fmaf(a.decay, before[i], w);
      else sWindow[j - G] = w;
    }
    j0 += kSlotsAhead * (kThreads / kSumHeads);
    if (j0 - tid / kSumHeads >= entries) break;  // (the same for the whole workgroup)
  }
  __syncthreads();
  if (tid == 0) {
    float w = 0.0f;
    for (int i = 0; i < n_win; ++i) w += sWindow[i];
    a.mass_out[at + G] = a.mass != nullptr ? fmaf(a.decay, a.mass[at + G], w) : w;
  }
}

}  // namespace

int launch_decode_mass(const MassCall& a, hipStream_t stream) {
  const dim3 grid((unsigned)((long long)a.cache.B * a.cache.H_kv * a.splits));
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  void (*kernel)(MassCall) = a.cache.bits == 4 ? (a.gq > 4 ? (sliding ? decode_mass_kernel<2, true, 4> : decode_mass_kernel<2, false, 4>)
                                                           : (sliding ? decode_mass_kernel<1, true, 4> : decode_mass_kernel<1, false, 4>))
                                               : (a.gq > 4 ? (sliding ? decode_mass_kernel<2, true, 2> : decode_mass_kernel<2, false, 2>)
                                                           : (sliding ? decode_mass_kernel<1, true, 2> : decode_mass_kernel<1, false, 2>));
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
