// One decode step that also accumulates what attention weight every group of tokens has received.
//
// The walk over the packed cache is that of kvlinc_windowed.hip without a window (shared in kvlinc_decode_parts.h): codes go to the matrix cores as
// FP4, weights as three FP8 terms, zero-points exact, all query heads of a KV head share one pass.  Weights are results here, so query times key scale
// has four terms (2^-16 of each product, see qk_phase), in the row of the matrix instruction that is spare.
// A weight is known only when the whole context has been seen.  So every wave leaves, for each group and head, its reference and its sum of weights, 64
// bytes a group beside the 9216 or 17408 it reads; and who joins the splits of a pair, and so knows the maximum M and the sum L of every head, makes
//     mass[j] = decay mass[j] + sum over heads of 2^(reference - M) sum / L,
// always in the same order.  No second pass over keys, no second launch.
// Bound: bytes of the groups.  32 sequences of 32k tokens, 7 heads, 4 bits: 117.8 us, 4.9 TB/s; of 16k to 32k 97 to 99, 4.5; 16 of 8k, 2 bits: 22.3 us, 3.6 TB/s,
// of which the chain of counters, first record, arrival, join and mass takes 6; one of 300 tokens: 8.4 us, the host's calls.  (The walk of few-row
// attention, which unpacks the codes for binary16 products: 119.5 for the 97, 28 for the 22.3.  Some 512 workgroups, two a compute unit; with 768 or
// 1024 16 of 8k take 22.1 and 26.  At 2 bits and up to 4 heads a unit has room for three, which serves batches of more pairs than 512: 736 of up to 900 tokens
// 17.3 us for 23.1, 800 of 1500 29 for 31.7.)  That room costs <1, *, 2> two registers' spills outside its loop (12 bytes a lane); <2, false, 4> and
// <2, true, 4> spill 11 and 18 in it (48 and 68 bytes a lane, 6 MB of the 4-bit call's writes).
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_decode_parts.h"
#include "kvlinc_join.h"

namespace kvlinc {
namespace {

constexpr int kHalfMirror = 0x141;  // row_half_mirror: lane 7 - i of every 8
constexpr int kSumHeads = 8;    // pairs {reference, sum} of a slot
constexpr int kShare = 32;     // tokens of the window a wave takes, with a slot of their own
constexpr int kSlotsAhead = 4;  // slots of a lane requested together

// {reference, sum} of a head: a store past the caches that are not coherent across the chip.
__device__ __forceinline__ void put_sum(unsigned long long* at, float reference, float sum) { st_coherent2(reinterpret_cast<float*>(at), reference, sum); }

// ---- which sequence and split a workgroup has ----
__device__ __forceinline__ int wave_sum(int v) {
  uint32_t u = (uint32_t)v;
  u += dpp_u<kRowRor1>(u);
  u += dpp_u<kRowRor2>(u);
  u += dpp_u<kRowRor4>(u);
  u += dpp_u<kRowRor8>(u);
  auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = a[0] + a[1];
  auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_amdgcn_readfirstlane((int)(b[0] + b[1]));
}
__device__ __forceinline__ int quotient_up(int n, int d) { return (int)((float)(n + d - 1) / (float)d); }  // (exact below 2^24)
struct Part {
  int b, split, splits;
  int before;  // splits of the sequences ahead, with room for those that a pair does not use
  int room;    // of the pair
};
// The sequences are cut into splits of the same number of groups a wave, the smallest with which the workgroups suffice: `units`, B at least, a KV head.  A
// lane a sequence; more than 64 of them are cut into as many splits each, and with no more workgroups than sequences every pair has one.  False: this
// workgroup has none.  (32 sequences of 16k to 32k tokens 108 us with four splits each, 96.8 so; of equal lengths nothing is lost.)
__device__ __forceinline__ bool part_of(const kvlinc_cache& c, int units, int unit, int lane, Part& p) {
  const int most = units / c.B;
  if (units == c.B || c.B == 1 || c.B > 64) {
    p.b = unit / most;
    p.split = unit - p.b * most;
    p.before = p.b * most;
    p.room = most;
    if (p.b >= c.B) return false;
    p.splits = max(1, min(most, (lengths_of(c, p.b).groups() + kWaves - 1) / kWaves));
    return p.split < p.splits;
  }
  const int groups = lane < c.B ? (c.n_quant[min(lane, c.B - 1)] + kGroup - 1) / kGroup : 0;
  const uint32_t in_row = row_umax((uint32_t)groups);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, (uint32_t)__builtin_amdgcn_readlane((int)in_row, 16 * i));
  const auto splits_at = [&](int rounds) __attribute__((always_inline)) {
    return lane < c.B ? max(1, min(kMaxContextSplits, quotient_up(groups, kWaves * rounds))) : 0;
  };
  int low = max(1, quotient_up(wave_sum(groups), kWaves * units)), high = max(low, quotient_up((int)top, kWaves * most));
  while (low < high) {
    const int mid = (low + high) / 2;
    if (wave_sum(splits_at(mid)) <= units) high = mid;
    else low = mid + 1;
  }
  const int splits = splits_at(high);
  int upto = splits;  // summed over the lanes up to this one
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, true);  // (the lane 1, 2, 4, 8 before it in its row of 16)
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, true);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, true);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, true);
  const int row = lane >> 4, r0 = __builtin_amdgcn_readlane(upto, 15), r1 = __builtin_amdgcn_readlane(upto, 31), r2 = __builtin_amdgcn_readlane(upto, 47);
  upto += (row > 0 ? r0 : 0) + (row > 1 ? r1 : 0) + (row > 2 ? r2 : 0);
  p.b = __popcll(__builtin_amdgcn_ballot_w64(upto <= unit));
  if (p.b >= c.B) return false;
  p.splits = p.room = __builtin_amdgcn_readlane(splits, p.b);
  p.before = __builtin_amdgcn_readlane(upto, p.b) - p.splits;
  p.split = unit - p.before;
  return true;
}

// Grid, one-dimensional: KV heads fastest, then what part_of shares out.
template <int NB, bool SLIDING, int BITS>
__global__ __launch_bounds__(kThreads, NB == 1 && BITS == 2 ? 3 : 2) void decode_mass_kernel(MassCall a) {
  constexpr int kCombine = 2 * kWaves * NB * 4 + kWaves * NB * 4 * kHeadDim, kRecordWords = Rec<BITS>::kWords, kTerms = 4;
  __shared__ __align__(16) float lds[kCombine + kWaves * 2 * kExWords];
  uint32_t (*ex)[2 * kExWords] = reinterpret_cast<uint32_t (*)[2 * kExWords]>(lds + kCombine);
  __shared__ float sRowM[kSumHeads], sRowL[kSumHeads];
  __shared__ int sLast;
  static_assert(kWaves * 2 * kExWords >= kThreads / 16 * kMaxContextSplits, "weights of the join");
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x / c.H_kv, head_kv = blockIdx.x - unit * c.H_kv, gq = a.gq;
  Part mine;
  if (!part_of(c, a.units, unit, lane, mine)) return;
  const int split = mine.split, n_splits = mine.splits, bh = mine.b * c.H_kv + head_kv;
  const Lengths len = lengths_of(c, mine.b);
  const int G = len.groups();
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
  const long long part0 = ((long long)mine.before * c.H_kv + (long long)head_kv * mine.room) * gq;
  const __amdgpu_buffer_rsrc_t part = buffer_of(a.part + (direct ? 0 : part0 * kPartStride), direct ? 0 : (long long)gq * n_splits * kPartBytes);
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
      const int place = (h * n_splits + split) * kPartBytes;
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
      join_row(part, h * n_splits * kPartBytes, n_splits, reinterpret_cast<float*>(&ex[0][0]) + kMaxContextSplits * h, lane, o, L, M);
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
  const dim3 grid((unsigned)((long long)a.units * a.cache.H_kv));
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  void (*kernel)(MassCall) = a.cache.bits == 4 ? (a.gq > 4 ? (sliding ? decode_mass_kernel<2, true, 4> : decode_mass_kernel<2, false, 4>)
                                                           : (sliding ? decode_mass_kernel<1, true, 4> : decode_mass_kernel<1, false, 4>))
                                               : (a.gq > 4 ? (sliding ? decode_mass_kernel<2, true, 2> : decode_mass_kernel<2, false, 2>)
                                                           : (sliding ? decode_mass_kernel<1, true, 2> : decode_mass_kernel<1, false, 2>));
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
