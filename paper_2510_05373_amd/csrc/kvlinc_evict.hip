// Eviction: which groups of a (sequence, KV head) stay, by their mass, and their records moved together.
//
// A group's key is an unsigned number that orders like its mass.  Caches of up to 512 or 256 groups: one launch.  Every workgroup selects for itself, in one wave
// that holds all keys of the pair: the largest threshold that enough keys reach is found bit by bit from the top, a comparison and a count of lanes for
// every 64 keys, no memory and no barrier; those above it stay, and of those equal to it the first ones.  Nothing that it reads (mass, counters) is
// written before all workgroups of the pair, or the sequence, have read it: whoever is the last to say so writes.  Larger caches: a launch before has
// a workgroup for each pair that finds the threshold by four counts of the keys' bits, 8 at a time, five reads of the mass, and leaves the list of what stays.
// Into another cache: a wave a record.  In place: a lane has 16 bytes of every record of a pair, and moves them from slot to slot in order.  A slot's
// source is never below it, so what the lane reads has not been written yet, whatever other lanes have done: no workgroup waits for another.
// Bound: bytes of the records that move, in and out: 128 pairs, 64 of 256 groups each, 4 bits, 300 MB: 59.7 us, what a copy takes; 128 pairs, 2k tokens of 8k:
// 11.2 us; one chat, 16 of 17 groups: 9.4 us, the host's call, of which the kernel takes 5.3, a chain of counters and mass, selection, record.  (With a
// launch of its own to select 68.9, 16.7 and 12.9; with what is written once ahead of the moves 15.0 for the 11.2.)  Caches of more groups pay for the
// launch that selects: 256 pairs of 1000 groups, 32 kept, 45 us, a copy 30.  In place few pairs have few waves, 9 or 17 each, every one a chain of
// loads and stores, 16 slots at a time: 8 pairs that all close up behind their second group, from a graph, 16 slots 5.0 us, 64 8.5, 511 40 (into another
// cache 17.9, a copy 14.8), 2 pairs of 511 38 (9.5, 3.7); 128 pairs, 64 of 256 groups at 4 bits 66 (60.6, 55.9).
#include <hip/hip_runtime.h>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_codes.h"

namespace kvlinc {
namespace {

constexpr int kSelectThreads = 256, kSelectWaves = kSelectThreads / 64;

// Orders like the mass: of two zeros neither is larger; what is not a number is below everything.
__device__ __forceinline__ uint32_t key_of(float mass) {
  if (mass != mass) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, mass + 0.0f);  // (-0 becomes 0)
  return (u >> 31) != 0 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictCall a) {
  __shared__ uint32_t sBins[256];
  __shared__ uint32_t sThreshold, sNeed;
  __shared__ int sKept[kSelectWaves], sTied[kSelectWaves], sFirst[kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long pair = blockIdx.x;
  const int b = (int)(pair / a.from.H_kv);
  const Lengths len = lengths_of(a.from, b);
  const int n = len.groups();
  const float* mass = a.mass + pair * (a.from.max_groups + 1);
  float* mass_out = a.mass_out + pair * (a.to.max_groups + 1);
  const int cut = n > a.limit ? a.keep : n, newest = n - a.last;

  // key and number of those with it that stay, among the groups a.first .. newest - 1
  uint32_t threshold = 0, need = 0;
  if (n > a.limit) {
    need = a.keep - a.first - a.last;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kSelectThreads) sBins[i] = 0;
      __syncthreads();
      for (int j = a.first + tid; j < newest; j += kSelectThreads) {
        const uint32_t key = key_of(mass[j]);
        if (shift == 24 || key >> (shift + 8) == threshold >> (shift + 8)) atomicAdd(&sBins[key >> shift & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {  // bins from the top: lane i has 255 - 4 i and the three below
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = sBins[255 - 4 * lane - i]; sum += c[i]; }
        uint32_t upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const uint32_t v = __shfl_up(upto, d);
          upto += lane >= d ? v : 0u;
        }
        uint32_t above = upto - sum;
        // (with nothing to choose, need = 0: the top bin of the first lane, nothing is above it)
        const bool here = need == 0 ? lane == 0 : above < need && upto >= need;
        if (here) {
          int i = 0;
          while (i < 3 && above + c[i] < need) above += c[i++];
          sThreshold = threshold | (uint32_t)(255 - 4 * lane - i) << shift;
          sNeed = need - above;
        }
      }
      __syncthreads();
      threshold = sThreshold;
      need = sNeed;
    }
  }

  // the list, kSelectThreads groups at a time
  int32_t* source = a.source + pair * a.stride;
  int kept = 0, tied = 0, first_moved = cut;
  const float window = mass[n];
  __syncthreads();
  for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
    const int j = j0 + tid;
    const float m = j < n ? mass[j] : 0.0f;
    const bool fixed = n <= a.limit || j < a.first || j >= newest;
    const uint32_t key = key_of(m);
    const bool tie = j < n && !fixed && key == threshold;
    const uint64_t ties = __builtin_amdgcn_ballot_w64(tie);
    if (lane == 0) sTied[wave] = __popcll(ties);
    __syncthreads();
    int before = tied;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
      before += w < wave ? sTied[w] : 0;
      tied += sTied[w];
    }
    before += __popcll(ties & ((1ull << lane) - 1));
    const bool stays = j < n && (fixed || key > threshold || (tie && (uint32_t)before < need));
    const uint64_t all = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) sKept[wave] = __popcll(all);
    __syncthreads();  // (and all of these groups' mass has been read: a slot it goes to is none of a later group)
    int slot = kept;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
      slot += w < wave ? sKept[w] : 0;
      kept += sKept[w];
    }
    slot += __popcll(all & ((1ull << lane) - 1));
    if (stays) {
      source[slot] = j;
      mass_out[slot] = m;
      if (a.kept != nullptr) a.kept[pair * a.to.max_groups + slot] = j;
      if (slot != j) first_moved = min(first_moved, slot);
    }
  }
  for (long long j = cut + tid; j <= a.to.max_groups; j += kSelectThreads) mass_out[j] = j == cut ? window : 0.0f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) first_moved = min(first_moved, __shfl_xor(first_moved, d));
  if (lane == 0) sFirst[wave] = first_moved;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) first_moved = min(first_moved, sFirst[w]);
    a.count[2 * pair] = cut;
    a.count[2 * pair + 1] = first_moved;
  }
}

// ---- selection by one wave ----
// BLOCKS: of 64 keys; 1, 4 or 8, as few as the cache has room for (0: a launch before has selected).
template <int BLOCKS>
struct Choice {
  int n, cut, first_moved;  // groups, how many stay, the first slot with another group than before (cut: none)
  float mass[BLOCKS + 1];  // of group 64 k + lane (n: the window's)
  uint64_t stay[BLOCKS];
};
template <int BLOCKS>
__device__ __forceinline__ void choose(Choice<BLOCKS>& c, const EvictCall& a, long long pair, int lane) {
  const float* mass = a.mass + pair * (a.from.max_groups + 1);
  const int most = (int)a.from.max_groups;
#pragma unroll
  for (int k = 0; k <= BLOCKS; ++k) c.mass[k] = 64 * k <= most ? mass[min(64 * k + lane, most)] : 0.0f;
  c.n = lengths_of(a.from, (int)(pair / a.from.H_kv)).groups();
  const int n = c.n, newest = n - a.last;
  c.cut = n > a.limit ? a.keep : n;
  c.first_moved = c.cut;
  if (n <= a.limit) {
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) c.stay[k] = __builtin_amdgcn_ballot_w64(64 * k + lane < n);
    return;
  }
  const auto of_choice = [&](int j) __attribute__((always_inline)) { return j >= a.first && j < newest; };
  uint32_t key[BLOCKS];  // (0, which counts reach nowhere, for the first groups and the newest)
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k) key[k] = of_choice(64 * k + lane) ? key_of(c.mass[k]) : 0u;
  const auto reaching = [&](uint32_t t /* > 0 */) __attribute__((always_inline)) {
    int count = 0;
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      if (64 * k >= n) break;
      count += __popcll(__builtin_amdgcn_ballot_w64(key[k] >= t));
    }
    return count;
  };
  const int need = a.keep - a.first - a.last;
  uint32_t t = 0;
  bool exact = false;  // just as many keys as needed reach t
  int bit = 31;
  for (; bit >= 0 && need > 0 && !exact; --bit) {
    const int count = reaching(t | 1u << bit);
    if (count >= need) t |= 1u << bit;
    exact = count == need;
  }
  // (t is the key of the last that stays, or between it and the next; keys equal to t: all stay, or the first ones)
  int ties = exact ? n : need <= 0 ? 0 : need - (t == ~0u ? 0 : reaching(t + 1));
  bool whole = true;
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k) {
    c.stay[k] = 0;
    if (64 * k >= n) continue;
    const int j = 64 * k + lane;
    const bool tie = of_choice(j) && key[k] == t;
    const uint64_t equal = __builtin_amdgcn_ballot_w64(tie);
    const bool chosen = need > 0 && (key[k] > t || (tie && (int)__popcll(equal & ((1ull << lane) - 1)) < ties));
    c.stay[k] = __builtin_amdgcn_ballot_w64(j < a.first || (j >= newest && j < n) || chosen);
    ties -= (int)__popcll(equal);
    if (whole && c.stay[k] != ~0ull) {
      whole = false;
      c.first_moved = min(c.cut, 64 * k + __builtin_ctzll(~c.stay[k]));
    }
  }
}
template <int BLOCKS>
__device__ __forceinline__ void list_of(const Choice<BLOCKS>& c, int lane, uint16_t* list /* LDS */) {
  int kept = 0;
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k) {
    if (64 * k >= c.n) break;
    if ((c.stay[k] >> lane & 1) != 0) list[kept + __popcll(c.stay[k] & ((1ull << lane) - 1))] = (uint16_t)(64 * k + lane);
    kept += __popcll(c.stay[k]);
  }
}
// The mass that goes with what is kept, and the list for the caller.
template <int BLOCKS>
__device__ __forceinline__ void put_masses(const Choice<BLOCKS>& c, const EvictCall& a, long long pair, int lane) {
  float* mass_out = a.mass_out + pair * (a.to.max_groups + 1);
  int kept = 0;
#pragma unroll
  for (int k = 0; k <= BLOCKS; ++k) {
    const int j = 64 * k + lane;
    if (64 * k > c.n) break;
    if (j == c.n) mass_out[c.cut] = c.mass[k];
    if (k == BLOCKS) break;
    const uint64_t stay = c.stay[k < BLOCKS ? k : 0];
    if ((stay >> lane & 1) != 0) {
      const int slot = kept + __popcll(stay & ((1ull << lane) - 1));
      mass_out[slot] = c.mass[k];
      if (a.kept != nullptr) a.kept[pair * a.to.max_groups + slot] = j;
    }
    kept += __popcll(stay);
  }
  for (long long j = c.cut + 1 + lane; j <= a.to.max_groups; j += 64) mass_out[j] = 0.0f;
}

// Counters of a sequence, by one thread, when everybody has read those of before.
__device__ __forceinline__ void commit(const EvictCall& a, int b, int cut) {
  const Lengths len = lengths_of(a.from, b);
  const int dropped = (len.groups() - cut) * kGroup;
  if (a.offset_out != nullptr) a.offset_out[b] = (a.offset != nullptr ? a.offset[b] : 0) + dropped;
  a.to.n_quant[b] = len.nq - dropped;
  a.to.n_res[b] = len.nr;
}

// What is written once: by a pair's workgroup `first`, or, where it is written over what the others read, by the last of the pair's `workgroups` to say that
// they have read it, and of the sequence's last ones by the last.  The counters that tell are the cache's own, zero before and after: of a
// pair, and in the upper half of the first pair's of the sequence, one for each of its pairs.
__device__ __forceinline__ int arrive(const EvictCall& a, long long pair, int lane) {
  int before = 0;
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // (mass and counters have been read)
  if (lane == 0 && a.counted) before = __hip_atomic_fetch_add(a.to.split_done + pair, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  return before;
}
template <int BLOCKS>
__device__ __forceinline__ void write_once(const Choice<BLOCKS>& c, const EvictCall& a, long long pair, int lane, bool first, int before, int workgroups) {
  if (a.counted ? (__builtin_amdgcn_readfirstlane(before) & 0xffff) != workgroups - 1 : !first) return;
  put_masses(c, a, pair, lane);
  const int heads = a.from.H_kv;
  const long long sequence = pair / heads;
  if (lane != 0) return;
  if (!a.counted) {
    if (pair % heads == 0) commit(a, (int)sequence, c.cut);
    return;
  }
  __hip_atomic_fetch_add(a.to.split_done + pair, -workgroups, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  const int others = __hip_atomic_fetch_add(a.to.split_done + sequence * heads, 1 << 16, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM) >> 16;
  if (others != heads - 1) return;
  __hip_atomic_fetch_add(a.to.split_done + sequence * heads, -(heads << 16), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  commit(a, (int)sequence, c.cut);
}

// Into another cache.  Grid: pairs in x, workgroups of a pair in y; a wave takes records, and, with the same number of 16-byte runs at a time, the window.
constexpr int kMoveWaves = 4;
// Stores past the caches from so many bytes on: 144 MB of 4-bit records 70.4 -> 59.7 us, of 2-bit ones 75.6 -> 72.9; 72 MB of these 35.5 -> 38.9, 21 MB
// 11.2 -> 11.9.  In place 136 MB 69.9 -> 64.2.
constexpr long long kStreamedBytes = 96ll << 20;
template <int BITS, int BLOCKS, bool STREAMED>
__global__ __launch_bounds__(64 * kMoveWaves) void move_kernel(EvictCall a) {
  constexpr int kRuns = Rec<BITS>::kWords / 4 / 64;
  static_assert(Rec<BITS>::kWords % 256 == 0, "whole runs of every lane");
  __shared__ uint16_t sList[BLOCKS == 0 ? 1 : 64 * BLOCKS];
  __shared__ int sCut;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long long pair = blockIdx.x;
  const int runs = a.from.R * (kHeadDim * 2 / 16), pieces = (runs + 64 * kRuns - 1) / (64 * kRuns);  // of the window's keys, and of its values
  int cut = 0;
  const auto units = [&]() __attribute__((always_inline)) {
    for (int u = blockIdx.y * kMoveWaves + wave; u < 2 * pieces + cut; u += gridDim.y * kMoveWaves) {
      const u32x4_t* src;
      u32x4_t* dst;
      int left = 64 * kRuns;
      if (u >= 2 * pieces) {
        const int slot = u - 2 * pieces;
        const int from = BLOCKS == 0 ? a.source[pair * a.stride + slot] : (int)sList[slot];
        src = reinterpret_cast<const u32x4_t*>(a.from.groups + (pair * a.from.max_groups + from) * Rec<BITS>::kWords);
        dst = reinterpret_cast<u32x4_t*>(a.to.groups + (pair * a.to.max_groups + slot) * Rec<BITS>::kWords);
      } else {
        const bool keys = u < pieces;
        const int at = (keys ? u : u - pieces) * 64 * kRuns;
        src = reinterpret_cast<const u32x4_t*>(keys ? a.from.k_res : a.from.v_res) + pair * runs + at;
        dst = reinterpret_cast<u32x4_t*>(keys ? a.to.k_res : a.to.v_res) + pair * runs + at;
        left = min(left, runs - at);
      }
      u32x4_t v[kRuns];
#pragma unroll
      for (int i = 0; i < kRuns; ++i)
        if (64 * i + lane < left) v[i] = __builtin_nontemporal_load(src + 64 * i + lane);
#pragma unroll
      for (int i = 0; i < kRuns; ++i) {
        if (64 * i + lane >= left) continue;
        if constexpr (STREAMED) __builtin_nontemporal_store(v[i], dst + 64 * i + lane);
        else dst[64 * i + lane] = v[i];
      }
    }
  };
  if constexpr (BLOCKS == 0) {
    cut = a.count[2 * pair];
    if (tid == 0 && blockIdx.y == 0 && pair % a.from.H_kv == 0) commit(a, (int)(pair / a.from.H_kv), cut);
    units();
  } else {
    Choice<BLOCKS> c;
    int before = 0;
    if (wave == 0) {
      choose(c, a, pair, lane);
      before = arrive(a, pair, lane);
      list_of(c, lane, sList);
      if (lane == 0) sCut = c.cut;
    }
    __syncthreads();
    cut = __builtin_amdgcn_readfirstlane(sCut);
    units();
    if (wave == 0) write_once(c, a, pair, lane, blockIdx.y == 0, before, gridDim.y);
  }
}

// In place.  Grid: pairs in x, waves of 64 runs of 16 bytes of a record in y.
constexpr int kAhead = 16;  // loads of a lane under way
template <int BITS, int BLOCKS, bool STREAMED>
__global__ __launch_bounds__(64) void close_up_kernel(EvictCall a) {
  constexpr int kVectors = Rec<BITS>::kWords / 4;
  static_assert(kVectors % 64 == 0, "grid");
  __shared__ uint16_t sList[BLOCKS == 0 ? 1 : 64 * BLOCKS];
  const int lane = threadIdx.x, at = blockIdx.y * 64 + lane;
  const long long pair = blockIdx.x;
  u32x4_t* base = reinterpret_cast<u32x4_t*>(a.to.groups + pair * a.to.max_groups * Rec<BITS>::kWords) + at;
  const auto move = [&](int first, int cut) __attribute__((always_inline)) {
    const int32_t* source = a.source + pair * a.stride;
    for (int j0 = first; j0 < cut; j0 += kAhead) {
      u32x4_t v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int slot = min(j0 + i, cut - 1);
        const u32x4_t* from = base + (long long)(BLOCKS == 0 ? source[slot] : (int)sList[slot]) * kVectors;
        v[i] = STREAMED ? __builtin_nontemporal_load(from) : *from;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (j0 + i >= cut) continue;
        if constexpr (STREAMED) __builtin_nontemporal_store(v[i], base + (long long)(j0 + i) * kVectors);
        else base[(long long)(j0 + i) * kVectors] = v[i];
      }
    }
  };
  if constexpr (BLOCKS == 0) {
    const int cut = a.count[2 * pair];
    if (at == 0 && pair % a.from.H_kv == 0) commit(a, (int)(pair / a.from.H_kv), cut);
    move(a.count[2 * pair + 1], cut);
  } else {
    Choice<BLOCKS> c;
    choose(c, a, pair, lane);
    const int before = arrive(a, pair, lane);
    if (c.first_moved < c.cut) {
      list_of(c, lane, sList);
      __syncthreads();
      move(c.first_moved, c.cut);
    }
    write_once(c, a, pair, lane, blockIdx.y == 0, before, gridDim.y);
  }
}

template <int BITS, int BLOCKS>
void launch_moves(const EvictCall& a, hipStream_t stream) {
  const unsigned pairs = (unsigned)(a.from.B * a.from.H_kv);
  if (a.in_place) {
    const long long records = a.keep < a.from.max_groups ? a.keep : a.from.max_groups;
    const bool streamed = (long long)pairs * records * Rec<BITS>::kWords * 4 >= kStreamedBytes;
    hipLaunchKernelGGL((streamed ? close_up_kernel<BITS, BLOCKS, true> : close_up_kernel<BITS, BLOCKS, false>), dim3(pairs, Rec<BITS>::kWords / 4 / 64), dim3(64), 0, stream, a);
  } else {
    const long long records = a.limit < a.from.max_groups ? a.limit : a.from.max_groups;
    const long long units = records + 2 * ((a.from.R * kHeadDim * 2 + Rec<BITS>::kWords * 4 - 1) / (Rec<BITS>::kWords * 4));
    const long long all = (units + kMoveWaves - 1) / kMoveWaves, most = 16384 / pairs;
    const dim3 grid(pairs, (unsigned)(all < most ? all : most < 1 ? 1 : most));
    const bool streamed = (long long)pairs * units * Rec<BITS>::kWords * 4 >= kStreamedBytes;
    hipLaunchKernelGGL((streamed ? move_kernel<BITS, BLOCKS, true> : move_kernel<BITS, BLOCKS, false>), grid, dim3(64 * kMoveWaves), 0, stream, a);
  }
}

}  // namespace

int launch_evict(const EvictCall& a, hipStream_t stream) {
  if (evicts_in_one_launch(a.from)) {
    if (a.from.max_groups <= 64) a.from.bits == 2 ? launch_moves<2, 1>(a, stream) : launch_moves<4, 1>(a, stream);
    else if (a.from.max_groups <= 256) a.from.bits == 2 ? launch_moves<2, 4>(a, stream) : launch_moves<4, 4>(a, stream);
    else launch_moves<2, 8>(a, stream);  // (at 4 bits there are no more)
    return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
  }
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)(a.from.B * a.from.H_kv)), dim3(kSelectThreads), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  a.from.bits == 2 ? launch_moves<2, 0>(a, stream) : launch_moves<4, 0>(a, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
