// Eviction: which groups of a (sequence, KV head) stay, by their mass, and their records moved together.
//
// Two launches.  The first has a workgroup for each pair: the mass of the m-th largest group is found by four counts of its bits, 8 at a time from the
// top (as an unsigned number that orders like the mass), so that any number of groups takes five reads of their mass; those above it stay, and of those
// equal to it the first ones.  It writes the list of what stays, in order, and the mass that goes with it.  The second moves records.  Into another
// cache: a workgroup a record.  In place: a lane has 16 bytes of every record of a pair, and moves them from slot to slot in order.  A slot's
// source is never below it, so what the lane reads has not been written yet, whatever other lanes have done: no workgroup waits for another.
// Bound: bytes of the records that move, in and out.
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

// Counters of a sequence, by one thread of its first KV head: what the first launch has read may change now.
__device__ __forceinline__ void commit(const EvictCall& a, int b, int cut) {
  const Lengths len = lengths_of(a.from, b);
  const int dropped = (len.groups() - cut) * kGroup;
  if (a.offset_out != nullptr) a.offset_out[b] = (a.offset != nullptr ? a.offset[b] : 0) + dropped;
  a.to.n_quant[b] = len.nq - dropped;
  a.to.n_res[b] = len.nr;
}

// Into another cache.  Grid: pairs in x; in y, as many at a time as there are, the records, then the window: pieces of kPieceBytes of keys and of values.
constexpr int kMoveThreads = 192, kPieceBytes = 8192;
template <int BITS>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictCall a, int records, int pieces) {
  constexpr int kVectors = Rec<BITS>::kWords / 4;
  const int tid = threadIdx.x;
  const long long pair = blockIdx.x;
  const int cut = a.count[2 * pair];
  for (int y = blockIdx.y; y < records + 2 * pieces; y += gridDim.y) {
    const u32x4_t* src;
    u32x4_t* dst;
    int vectors = kVectors;
    if (y < records) {
      if (y >= cut) continue;
      const int from = a.source[pair * a.stride + y];
      src = reinterpret_cast<const u32x4_t*>(a.from.groups + (pair * a.from.max_groups + from) * Rec<BITS>::kWords);
      dst = reinterpret_cast<u32x4_t*>(a.to.groups + (pair * a.to.max_groups + y) * Rec<BITS>::kWords);
    } else {
      const int bytes = a.from.R * kHeadDim * 2, part = y - records, piece = part < pieces ? part : part - pieces;
      const long long at = pair * (bytes / 16) + piece * (kPieceBytes / 16);
      src = reinterpret_cast<const u32x4_t*>(part < pieces ? a.from.k_res : a.from.v_res) + at;
      dst = reinterpret_cast<u32x4_t*>(part < pieces ? a.to.k_res : a.to.v_res) + at;
      vectors = min(kPieceBytes, bytes - piece * kPieceBytes) / 16;
      if (part == 0 && tid == 0 && pair % a.from.H_kv == 0) commit(a, (int)(pair / a.from.H_kv), cut);
    }
    for (int i = tid; i < vectors; i += kMoveThreads) dst[i] = __builtin_nontemporal_load(src + i);
  }
}

// In place.  Grid: pairs in x, waves of 64 runs of 16 bytes of a record in y.
constexpr int kAhead = 16;  // loads of a lane under way
template <int BITS>
__global__ __launch_bounds__(64) void close_up_kernel(EvictCall a) {
  constexpr int kVectors = Rec<BITS>::kWords / 4;
  const int at = blockIdx.y * 64 + threadIdx.x;
  const long long pair = blockIdx.x;
  const int cut = a.count[2 * pair];
  if (at == 0 && pair % a.from.H_kv == 0) commit(a, (int)(pair / a.from.H_kv), cut);
  if (at >= kVectors) return;
  const int32_t* source = a.source + pair * a.stride;
  u32x4_t* base = reinterpret_cast<u32x4_t*>(a.to.groups + pair * a.to.max_groups * Rec<BITS>::kWords) + at;
  for (int j0 = a.count[2 * pair + 1]; j0 < cut; j0 += kAhead) {
    u32x4_t v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = base[(long long)source[min(j0 + i, cut - 1)] * kVectors];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (j0 + i < cut) base[(long long)(j0 + i) * kVectors] = v[i];
  }
}

template <int BITS>
void launch_moves(const EvictCall& a, hipStream_t stream) {
  const unsigned pairs = (unsigned)(a.from.B * a.from.H_kv);
  if (a.in_place) {
    hipLaunchKernelGGL((close_up_kernel<BITS>), dim3(pairs, (Rec<BITS>::kWords / 4 + 63) / 64), dim3(64), 0, stream, a);
  } else {
    const long long records = a.limit < a.from.max_groups ? a.limit : a.from.max_groups;
    const int pieces = (a.from.R * kHeadDim * 2 + kPieceBytes - 1) / kPieceBytes;
    const long long all = records + 2 * pieces, most = 32768 < (1 << 24) / pairs ? 32768 : (1 << 24) / pairs;
    hipLaunchKernelGGL((move_kernel<BITS>), dim3(pairs, (unsigned)(all < most ? all : most < 1 ? 1 : most)), dim3(kMoveThreads), 0, stream, a, (int)records, pieces);
  }
}

}  // namespace

int launch_evict(const EvictCall& a, hipStream_t stream) {
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)(a.from.B * a.from.H_kv)), dim3(kSelectThreads), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  a.from.bits == 2 ? launch_moves<2>(a, stream) : launch_moves<4>(a, stream);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
