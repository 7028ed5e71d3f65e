// Windowed decode: one query a sequence over the newest tokens and the first few, read directly from the packed cache.
//
// The arithmetic is that of the decode kernel (kvlinc_decode.hip; shared in kvlinc_decode_parts.h): codes go to the matrix cores as FP4, queries
// and weights as three FP8 terms, zero-points exact (EXACT_OFFSETS), all query heads of a KV head share one pass.  What differs is which groups are
// walked: those with sinks, then those from the window's first token on, numbered one after the other; tokens of a group at the border that are not
// seen have their scores taken out.  A sequence is cut into splits of these groups; the four waves of split 0 share the visible part of the fp16 window first.
// One launch; the splits are joined by the workgroup that arrives last at the pair's counter.
// Bound: bytes of the visible groups (64 sequences, window 4096, 2 bits: 29.4 us, 5.4 TB/s; 32 of 7 heads, window 8192, 4 bits: 32.8 us, 4.6 TB/s;
// with sliding values 1.9 and 3.5 us more); small windows: latency, a chain of counters, record, combine (and arrival, join): one sequence, window 1024:
// 7.3 us, 7.6 with the host's calls.
#include <hip/hip_runtime.h>

#include "kvlinc_decode_parts.h"
#include "kvlinc_join.h"

namespace kvlinc {
namespace {

// Tokens 16 n + jd of a group at position `at` that the query sees keep their scores.
template <int NB>
__device__ __forceinline__ void hide_tokens(float (&sc)[NB][8], int at, int low, int sinks, const Roles& lr) {
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const int pos = at + 16 * n + lr.jd;
    const bool seen = pos >= low || pos < sinks;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sc[nb][n] = seen ? sc[nb][n] : -INFINITY;
  }
}

// Grid, one-dimensional: (sequence, KV head) fastest, then the split.
template <int NB, bool SLIDING, int BITS>
__global__ __launch_bounds__(kThreads, BITS == 4 || (NB == 2 && SLIDING) ? 2 : 3) void windowed_kernel(ContextCall a) {
  constexpr int kCombine = 2 * kWaves * NB * 4 + kWaves * NB * 4 * kHeadDim, kRecordWords = Rec<BITS>::kWords;
  __shared__ __align__(16) float lds[kCombine + kWaves * 2 * kExWords];
  uint32_t (*ex)[2 * kExWords] = reinterpret_cast<uint32_t (*)[2 * kExWords]>(lds + kCombine);
  __shared__ int sLast;
  static_assert(kWaves * 2 * kExWords >= kThreads / 16 * kMaxContextSplits, "weights of the join");
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pairs = c.B * c.H_kv, split = blockIdx.x / pairs, bh = blockIdx.x - split * pairs, b = bh / c.H_kv, g = bh - b * c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int total = len.total(), low = window_low(total - 1, a.window);
  // (every group walked has a token that is seen: what the running maximum of the shared code needs)
  const int G = len.groups(), group_low = low < len.nq ? low / kGroup : G;
  const int n_sink = a.window > 0 ? min((int)(((long long)a.sinks + kGroup - 1) / kGroup), group_low) : 0;
  const int count = G - group_low + n_sink;
  // every workgroup of the pair comes to the same number: a split has a group for each wave
  const int n_splits = max(1, min(a.splits, (count + kWaves - 1) / kWaves));
  if (split >= n_splits) return;
  const long long row0 = (long long)b * c.H_q + (long long)g * gq;  // (one token a sequence: places are heads)
  auto group_of = [&](int it) { return it < n_sink ? it : it - n_sink + group_low; };

  const Roles lr = make_roles(lane, ex[wave]);
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * kRecordWords;
  GroupOrder order(n_splits, split, wave, BITS == 2 && n_splits > 1 ? 2 : 1);
  int rd = split == 0 ? order.skip : 0, idx = order.group(rd);
  KeyRegs<BITS> kr;
  ValueRegs<BITS> vr;
  if (idx < count) {
    const uint32_t* src = rec0 + (long long)group_of(idx) * kRecordWords;
    load_keys(kr, src, lr);
    load_values(vr, src, lr);
  }
  uint32_t qh[NB][4];  // q of the head this lane builds operands for (head 4 nb + ha, or the last one), channels c0 .. c0 + 7
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const uint4 raw = *reinterpret_cast<const uint4*>(a.q + (row0 + min(nb * 4 + lr.ha, gq - 1)) * kHeadDim + lr.c0);
    qh[nb][0] = raw.x; qh[nb][1] = raw.y; qh[nb][2] = raw.z; qh[nb][3] = raw.w;
  }
  // the spare term row of every head of the exchange regions reads as zero
#pragma unroll
  for (int k = 0; k < 4; ++k) ex[wave][(k >> 1) * kExWords + (2 * (k & 1) + (lane >> 5)) * kExHead + 96 + (lane & 31)] = 0u;
  lds_order();
  WaveState<NB> st;
  empty_state<NB>(st);
  if (split == 0) {  // slots from_slot .. of the window are visible, and those of sinks
    const int from_slot = min(max(low - len.nq, 0), len.nr), sink_slots = a.window > 0 ? a.sinks - len.nq : 0;
    const int w0 = sink_slots > 0 ? 0 : from_slot & ~3;
    const WindowShare sh = {w0 + 32 * wave, min(w0 + 32 * wave + 32, len.nr)};
    if (sh.first < sh.end && (sh.end > from_slot || sh.first < sink_slots)) {
      WindowRegs w;
      request_window(w, c, bh, sh, lr);
      window_part<NB>(w, qh, sh, lr, st, from_slot, sink_slots);
    }
  }
  const half_t* const v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  float (*sM)[NB * 4] = reinterpret_cast<float (*)[NB * 4]>(lds);
  float (*sL)[NB * 4] = reinterpret_cast<float (*)[NB * 4]>(lds + kWaves * NB * 4);
  float (*sAcc)[NB * 4][kHeadDim] = reinterpret_cast<float (*)[NB * 4][kHeadDim]>(lds + 2 * kWaves * NB * 4);
  // (the newest group is left to the code below where its tokens from n_res on take the window's values)
  const int plain = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup && count > 0 && group_of(count - 1) == G - 1 ? count - 1 : count;
  while (idx < plain) {
    const int gr = group_of(idx), at = gr * kGroup, next = order.group(++rd);
    const bool more = next < count;
    const uint32_t* src = rec0 + (long long)group_of(more ? next : idx) * kRecordWords;
    float sc[NB][8], off[NB], base[NB];
    qk_phase<NB, BITS, true>(kr, min(kGroup, len.nq - at), qh, lr, sc, off);
    if (more) load_keys(kr, src, lr);
    if (at < low && at + kGroup > a.sinks) hide_tokens<NB>(sc, at, low, a.sinks, lr);
    update_reference<NB>(sc, off, base, st, kSlack);
    pv_phase<NB, BITS>(vr, sc, base, lr, st);
    if (more) load_values(vr, src, lr);
    idx = next;
  }
  if (SLIDING && idx < count) {
    const int at = group_of(idx) * kGroup;
    float sc[NB][8], off[NB], base[NB];
    qk_phase<NB, BITS, true>(kr, kGroup, qh, lr, sc, off);
    if (at < low && at + kGroup > a.sinks) hide_tokens<NB>(sc, at, low, a.sinks, lr);
    update_reference<NB>(sc, off, base, st, kSlack);
    pv_phase<NB, BITS, true>(vr, sc, base, lr, st, len.nr);
    pv_window_tail<NB>(v_win, sc, base, len.nr, lr, st, lane, sAcc[wave]);
  }

  // ---- the waves joined; one (m, l, numerators) a head ----
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float l = row_allsum(st.l[nb]), pz = row_allsum(st.pz[nb]);
    const int h = nb * 4 + lr.hd;
    if (lr.jd == 0) { sM[wave][h] = st.m[nb]; sL[wave][h] = l; }
#pragma unroll
    for (int n = 0; n < 8; ++n) sAcc[wave][h][16 * n + lr.jd] = st.acc[nb][n] + pz;
  }
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
    } else {
      const int place = (h * a.splits + split) * kPartBytes;
      if ((lane & 15) == 0) store2(part, place, M, L);
      store4(part, place + 16 + 4 * ch, o[0], o[1], o[2], o[3]);
      store4(part, place + 32 + 4 * ch, o[4], o[5], o[6], o[7]);
    }
  }
  if (direct) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's results are where everybody sees them
  __syncthreads();
  if (tid == 0) sLast = __hip_atomic_fetch_add(c.split_done + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) == n_splits - 1;
  __syncthreads();
  if (!__builtin_amdgcn_readfirstlane(sLast)) return;
  if (h < gq) {
    float o[8], L, M;
    join_row(part, h * a.splits * kPartBytes, n_splits, reinterpret_cast<float*>(&ex[0][0]) + kMaxContextSplits * h, lane, o, L, M);
    finish_row(o, L, lane, a.out + (row0 + h) * kHeadDim);
  }
  if (tid == 0) c.split_done[bh] = 0;
}

}  // namespace

int launch_windowed(const ContextCall& a, hipStream_t stream) {
  const dim3 grid((unsigned)((long long)a.cache.B * a.cache.H_kv * a.splits));
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  void (*kernel)(ContextCall) = a.cache.bits == 4 ? (a.gq > 4 ? (sliding ? windowed_kernel<2, true, 4> : windowed_kernel<2, false, 4>)
                                                              : (sliding ? windowed_kernel<1, true, 4> : windowed_kernel<1, false, 4>))
                                                  : (a.gq > 4 ? (sliding ? windowed_kernel<2, true, 2> : windowed_kernel<2, false, 2>)
                                                              : (sliding ? windowed_kernel<1, true, 2> : windowed_kernel<1, false, 2>));
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
