// Prompt attention of many row blocks: the cached tokens that the call sees are dequantized once, to binary16 rows in the workspace (the
// read-back kernel, values in the rotated basis), and blocks of 256 query rows go over tiles of 64 raw tokens.
//
// Rows, products, softmax and schedule are those of kvlinc_prompt.hip; what differs is how a tile comes to LDS: as it lies in memory, [token]
// [128 channels], by loads that write LDS themselves, so that no wave spends a register or a vector instruction on it.  The value operand
// (rows = channels) comes out of the row-major tile by transposing LDS reads.
// What the keys' rounding to binary16 leaves comes with them (64 bytes of FP4 numbers and 4 of scales a token, see LowTile): 8k tokens over 24k
// took 3.7 ms without it, 4.05 with it, at a third of the error.
//
// Bound: the matrix and the vector phases, which take turns on a SIMD's two waves and are about as long; a long call also the power limit (8k tokens
// over 24k: 1.67 GHz).  8k over 24k, 4 heads, with 0.08 ms of correction and 0.05 of dequantizing: 3.97 to 4.22 ms by the card (0.92 to 0.98 PFLOP/s; a
// matrix product of 8192^3 from the library reaches 1.19); four prompts of 1700 to 4096 tokens 393 to 402 us (0.86), 340 without the softmax, 312 without
// the products; one of 700 tokens 30.6 us.
#include <hip/hip_runtime.h>

#include "kvlinc_tiles.h"

namespace kvlinc {
namespace {

// 16-byte chunks of a row are permuted by the row: chunk c of row r lies at c ^ flip(r).  Two patterns have to spread over the banks:
// the keys' reads take one chunk of 16 consecutive rows, the values' 64 bytes of four consecutive rows; the low two bits of the row
// choose among 64-byte pieces, the next two within one.
__device__ __forceinline__ int flip(int row) { return (row & 3) << 2 | ((row >> 2) & 3); }

constexpr int kDenseBuffers = 4;
constexpr int kTileBytes = kTileTokens * kHeadDim * 2;
struct DenseTiles {
  char k[kDenseBuffers][kTileBytes];
  char v[kDenseBuffers][kTileBytes];
  LowTile low[kDenseBuffers];
  uint32_t bad[kDenseBuffers][4];  // tokens 16 i .. 16 i + 15 whose values are not finite, a bit each (see look_over)
  uint32_t again;
};

// 1 KB from memory to LDS, 16 bytes a lane, in lane order from `lds` on.  (In assembly: the compiler would otherwise wait for the tile under
// way ahead of every LDS read that it cannot tell from it.  There is no register to write.  The waits are in landed(); a load that writes LDS needs one
// wait state after a scalar write of m0, which the compiler adds to its own code only.)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_words_to_lds(const void* base, uint32_t offset, uint32_t lds) {  // 4 bytes a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// All but the newest N of this wave's loads have arrived.
template <int N>
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

typedef short short4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2_t lds_transposed(const char* p) {
  typedef __attribute__((address_space(3))) short4_t* lds_ptr;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p)));
}

// S^T = K Q^T.  Rows i and 32 + i, chunks 2 k + h: k in address bits 5..7.
__device__ __forceinline__ void dense_scores(TileRows& st, const char* t, int lane) {
  const int i = lane & 31, base = i * 256 + 16 * ((lane >> 5) ^ flip(i));
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.s[tb][r] = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) st.s[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_operand(t, (base ^ (32 * k)) + 8192 * tb), st.q[k], st.s[tb], 0, 0, 0);
}
// O^T += V^T P^T.  A transposing read gives lane i of 16 element i % 4 of what lanes i / 4, 4 + i / 4, 8 + i / 4, 12 + i / 4 point at: lane l points at
// token 16 s + 8 u + 4 h + (l % 16) / 4 (h = l / 32), channels 32 cb + 16 ((l / 16) % 2) + 4 (l % 4) .. + 3.
__device__ __forceinline__ void dense_values(TileRows& st, const char* t, int lane) {
  const int h = lane >> 5, row = 4 * h + ((lane & 15) >> 2), chunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
  const int base = row * 256 + 16 * (chunk ^ flip(row)) + 8 * (lane & 1);
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) {
      const u32x2_t a = lds_transposed(t + ((base ^ (64 * cb)) + 4096 * s)), b = lds_transposed(t + ((base ^ (64 * cb) ^ 32) + 2048 + 4096 * s));
      st.acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(u32x4_t{a[0], a[1], b[0], b[1]}), st.p[s], st.acc[cb], 0, 0, 0);
    }
}
// Order of a matrix phase (see matrix_order): products of values take two reads each, those of scores one.
template <bool VALUES>
__device__ __forceinline__ void dense_order() {
  constexpr int kProducts = VALUES ? 32 : 16, kFirst = VALUES ? 12 : 6;
  __builtin_amdgcn_sched_group_barrier(0x100, kFirst, 0);
#pragma unroll
  for (int i = 0; i < kProducts; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (VALUES && i < 16 - kFirst / 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    else if (i < (VALUES ? 32 - kFirst / 2 : 16 - kFirst)) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}

// New values that are not finite must not reach rows that do not see them: 0 times such a value is not a number.  A block goes over its tiles without a
// look at that, and once more, looking at every new value, if one of its rows has not come out finite (finite values leave all sums far below binary32's
// largest number).  Looked at in the first place they took 1 to 4 % of a call (700 tokens 31.9 -> 33.4 us, four prompts of 1700 to 4096 395 -> 405); so it
// is 0.5 % (32.3; 397).  (The kernel that unpacks codes has them in registers on their way and looks at once: a second time cost its short calls 1.5 us.)
__device__ __forceinline__ bool rows_not_finite(const TileRows& st) {
  float z = st.l * 0.0f;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(st.acc[cb][r], 0.0f, z);
  return __builtin_amdgcn_ballot_w64(z != 0.0f) != 0;
}
// Whether some wave of the block has to; `word`: LDS, 0 since before the last barrier but one.  Ends with all waves at one place.
__device__ __forceinline__ bool some_wave(bool mine, uint32_t& word, int lane) {
  if (mine && lane == 0) word = 1;
  next_phase();
  return __builtin_amdgcn_readfirstlane(word) != 0;
}
// The second time over a block's tiles (see rows_not_finite): waves 0..3 look at 16 rows of new values each ahead of the tile's products, a quarter
// of a row a lane, put zeros in the place of what is not finite and note the token.
__device__ __forceinline__ void look_over(char* t, uint32_t& bad, int wave, int lane) {
  u32x4_t* row = reinterpret_cast<u32x4_t*>(t + 4096 * wave + 64 * lane);  // (which chunks they are does not matter)
  u32x4_t x[4];
  uint32_t here = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    x[c] = row[c];
#pragma unroll
    for (int i = 0; i < 4; ++i) here |= not_finite(x[c][i]);
  }
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(here != 0);
  uint32_t tokens = 0;
  if (lanes != 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) tokens |= (lanes >> (4 * i) & 15u) != 0 ? 1u << i : 0u;
    if (here != 0)
#pragma unroll
      for (int c = 0; c < 4; ++c) row[c] = u32x4_t{finite_or_zero(x[c][0]), finite_or_zero(x[c][1]), finite_or_zero(x[c][2]), finite_or_zero(x[c][3])};
  }
  if (lane == 0) bad = tokens;
}

// Rows of a sequence that holds more tokens than the workspace has rows for: zeros, and a bit in the status word.
__device__ __forceinline__ void refuse_rows(const ContextCall& a, const WaveRows& w, int split, int lane) {
  if (w.idle) return;
  if (lane == 0) atomicOr(a.cache.status, KVLINC_ST_BOUND);
  if (!w.mine) return;
  const int h = lane >> 5;
  auto clear = [&](void* row, int bytes) __attribute__((always_inline)) {
    for (int at = 16 * h; at < bytes; at += 32) *reinterpret_cast<uint4*>(static_cast<char*>(row) + at) = make_uint4(0, 0, 0, 0);
  };
  if (a.splits == 1) {
    clear(a.out + w.place * kHeadDim, kHeadDim * 2);
    return;
  }
  // (the join makes zeros of empty splits and an empty correction)
  float* dst = a.part + (w.place * a.splits + split) * kPartStride;
  clear(dst, kPartStride * 4);
  if (h == 0) dst[0] = -INFINITY;
  if (a.corr != nullptr) clear(a.corr + w.place * kPartStride, kPartStride * 4);
}

// Grid, one-dimensional: see place_of_block.
__global__ __launch_bounds__(kTileThreads, 2) void dense_kernel(ContextCall a, int blocks) {
  __shared__ __align__(1024) DenseTiles tiles;
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const BlockPlace at_block = place_of_block(a, blocks);
  const int split = at_block.split, bh = at_block.bh, block = at_block.block;
  const int b = bh / c.H_kv, kvh = bh - b * c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int T = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T;
  const int rows = T * gq, row0 = block * kTileRows;
  if (row0 >= rows) return;
  const int total = len.total();
  const WaveRows wr = wave_rows(a, b, kvh, rows, row0 + 32 * wave, total, lane);

  TileRows st;
  start_rows(st, a.q + wr.place * kHeadDim, lane);
  LowQuery low;
  if (total > 0) low = low_query(a.q + wr.place * kHeadDim, lane);

  // Tiles that some row of the block sees: of the new rows; of the sinks; of the tokens from `near` on.  Positions of the workspace's rows:
  // 0 .. near_row - 1 are the sinks' (tokens 0 ..), from near_row on the tokens from `near` on.
  const int last_i = min(row0 + kTileRows - 1, rows - 1) / gq, low_block = window_low(total + row0 / gq, a.window);
  const int new_from = a.sinks > total ? 0 : max(low_block - total, 0) / kTileTokens;
  const int n_new = last_i / kTileTokens + 1 - new_from;
  const int near = window_base(total, a.row_window), near_row = a.sink_rows;
  const int held = min(total, near + a.cached_rows - near_row);  // (all of them, unless the caller's bound was too low)
  if (held < total) {
    refuse_rows(a, wr, split, lane);
    return;
  }
  const int n_sink = (min(a.sinks, near) + kTileTokens - 1) / kTileTokens;
  const int near_from = a.sinks > near ? 0 : (min(low_block, held) - near) / kTileTokens;
  const int n_near = (held - near + kTileTokens - 1) / kTileTokens - near_from;
  const int n_tiles = n_new + n_sink + n_near;
  const int first = (int)((long long)n_tiles * split / a.splits), last = (int)((long long)n_tiles * (split + 1) / a.splits);

  const half_t* new_keys = a.k_new + (long long)bh * a.T * kHeadDim;
  const half_t* new_values = a.v_new + (long long)bh * a.T * kHeadDim;
  const half_t* old_keys = a.k_rows + (long long)bh * a.cached_rows * kHeadDim;
  const half_t* old_values = a.v_rows + (long long)bh * a.cached_rows * kHeadDim;
  const u32x4_t* low_rows = reinterpret_cast<const u32x4_t*>(a.k_low) + (long long)bh * a.cached_rows * 4;
  const uint32_t* low_scales = a.k_low_scale + (long long)bh * a.cached_rows;

  struct Tile { int at, row, count; bool fresh; };  // position of its first token, row in its source, tokens
  auto tile_of = [&](int it) {
    Tile t;
    t.fresh = it < n_new;
    if (t.fresh) {
      t.row = (new_from + it) * kTileTokens;
      t.at = total + t.row;
      t.count = min(T - t.row, kTileTokens);
    } else if (it < n_new + n_sink) {
      t.row = t.at = (it - n_new) * kTileTokens;
      t.count = min(held - t.at, kTileTokens);
    } else {
      const int r = (near_from + it - n_new - n_sink) * kTileTokens;
      t.row = near_row + r;
      t.at = near + r;
      t.count = min(held - t.at, kTileTokens);
    }
    return t;
  };
  // A wave brings rows 4 w .. 4 w + 3 and 32 + 4 w .. of the keys and of the values: lane l chunk l % 16 of row l / 16, taken from where the
  // permutation has it.  Rows beyond the tile's tokens take the last one's (they are masked).
  const uint32_t lds_k = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&tiles.k[0][0] + 1024 * wave;
  const uint32_t lds_v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&tiles.v[0][0] + 1024 * wave;
  const int my_row = 4 * wave + (lane >> 4), my_chunk = 16 * ((lane & 15) ^ flip(my_row));  // (flip(row + 32) is the same)
  // Of the low parts, waves 0..3 bring a quarter each, rows 16 w + l / 4, and waves 4..7 the scales (the same 256 bytes: their loads are as many).
  const uint32_t lds_low = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&tiles.low[0] + (wave < 4 ? 1024 * wave : (int)sizeof(tiles.low[0].k));
  const int low_row = wave < 4 ? 16 * wave + (lane >> 2) : lane, low_at = 16 * low_chunk(low_row, lane & 3);
  auto bring = [&](int it, int buffer) __attribute__((always_inline)) {
    const Tile t = tile_of(it);
    const half_t* keys = (t.fresh ? new_keys : old_keys) + (long long)t.row * kHeadDim;
    const half_t* values = (t.fresh ? new_values : old_values) + (long long)t.row * kHeadDim;
    const uint32_t o0 = 256 * min(my_row, t.count - 1) + my_chunk, o1 = 256 * min(my_row + 32, t.count - 1) + my_chunk;
    load_to_lds(keys, o0, lds_k + kTileBytes * buffer);
    load_to_lds(keys, o1, lds_k + kTileBytes * buffer + 8192);
    load_to_lds(values, o0, lds_v + kTileBytes * buffer);
    load_to_lds(values, o1, lds_v + kTileBytes * buffer + 8192);
    if (t.fresh) return;
    if (wave < 4) load_to_lds(low_rows + (long long)t.row * 4, 64 * min(low_row, t.count - 1) + low_at, lds_low + (int)sizeof(LowTile) * buffer);
    else load_words_to_lds(low_scales + t.row, 4 * min(low_row, t.count - 1), lds_low + (int)sizeof(LowTile) * buffer);
  };

  // Tile `first` + k lies in buffer k % 4.  Waves 0..3 bring theirs two tiles ahead of the softmax, waves 4..7, a phase behind them, three: all
  // of a tile is there when waves 0..3 take its keys, and what it is written over (four tiles before) has been read by all.
  const int n = last - first, behind = wave >> 2;
  bool rotated = first >= n_new, careful = false;
  if (tid == 0) tiles.again = 0;
#pragma unroll 1
  while (n > 0) {
    int to = 0;
#pragma unroll 1
    for (; to < 2 + behind && to < n; ++to) bring(first + to, to);
    landed<0>();
#pragma unroll
    for (int k = 0; k < 8; ++k) asm volatile("" : "+v"(st.q[k]));  // (and so has q, for the compiler's count)
    next_phase();
    if (behind) next_phase();
    if (!wr.idle) dense_scores(st, tiles.k[0], lane);
    if (!wr.idle && first >= n_new) low_scores(st, tiles.low[0], low, lane);
    next_phase();
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      // vector phase
      const int item = first + k;
      if (item == n_new && !rotated) {
        rotate_tile_rows(st, lane);
        rotated = true;
      }
      const bool more = to < n;
      if (more) {
        bring(first + to, to & 3);
        ++to;
      }
      const Tile t = tile_of(item);
      const bool live = wave_sees(wr, a, t.at, t.count);
      if (live) tile_weights(st, t.at, t.count, wave_masked(wr, a, t.at, t.count), wr.p, wr.low, a.sinks, lane);
      const bool look = careful && t.fresh;
      if (look && !behind) look_over(tiles.v[k & 3], tiles.bad[k & 3][wave], wave, lane);
      // the tile before the one just asked for
      if (!more) landed<0>();
      else if (first + to <= n_new) landed<4>();
      else landed<5>();
      next_phase();
      // matrix phase
      if (live) {
        dense_values(st, tiles.v[k & 3], lane);
        dense_scores(st, tiles.k[(k + 1) & 3], lane);  // (of the last tile: what the next buffer held; not used)
        dense_order<true>();
      } else if (!wr.idle) {
        dense_scores(st, tiles.k[(k + 1) & 3], lane);
        dense_order<false>();
      }
      // (a block of its own: one for both kinds of tiles in each of the above kept two copies of the accumulators)
      if (look) {
        const uint32_t(&b)[4] = tiles.bad[k & 3];
        const uint64_t bad = b[0] | (uint64_t)b[1] << 16 | (uint64_t)b[2] << 32 | (uint64_t)b[3] << 48;
        if (__builtin_amdgcn_readfirstlane((uint32_t)bad | (uint32_t)(bad >> 32)) != 0) spoil_rows(st, bad, t.at, wr.p, wr.low, a.sinks);
      }
      if (item + 1 >= n_new && !wr.idle) low_scores(st, tiles.low[(k + 1) & 3], low, lane);
      next_phase();
    }
    if (!behind) next_phase();
    if (careful || !some_wave(!wr.idle && rows_not_finite(st), tiles.again, lane)) break;
    careful = true;
    rotated = first >= n_new;
    start_rows(st, a.q + wr.place * kHeadDim, lane);
  }
  const bool in_cache_basis = total > 0 || a.splits > 1;
  if (in_cache_basis && !rotated) rotate_tile_rows(st, lane);
  store_results(st, a, wr, split, in_cache_basis, lane);
}

}  // namespace

int launch_dense(const ContextCall& a, hipStream_t stream) {
  // the cached tokens that some row sees, as rows: the sinks (if they lie apart), and what is near
  const int rc = launch_read_rows(a, stream);
  if (rc != KVLINC_OK) return rc;
  const int blocks = (int)(((long long)a.T * a.gq + kTileRows - 1) / kTileRows);
  const dim3 grid((unsigned)((long long)blocks * a.cache.B * a.cache.H_kv * a.splits));
  hipLaunchKernelGGL(dense_kernel, grid, dim3(kTileThreads), 0, stream, a, blocks);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  return a.splits > 1 ? launch_join(a, stream) : KVLINC_OK;
}

}  // namespace kvlinc
