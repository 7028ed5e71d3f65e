// Prompt attention of many rows: blocks of 256 query rows over tiles of 64 tokens that the whole workgroup shares through LDS.
//
// Rows of a (sequence, KV head) are (token i, head h) pairs, row = i gq + h, so that a block covers few tokens and all heads share the
// tiles and the causal border.  Eight waves have 32 rows each; a tile is fetched into registers while the one before is worked on, turned
// into binary16 (packed codes: once for the 256 rows) and put into the other half of the LDS, one barrier a tile.
//
// Both products run on v_mfma_f32_32x32x16_f16, transposed: S^T = K Q^T (rows = tokens, columns = query rows) and O^T = V^T P^T (rows =
// channels), so that a lane holds one query row throughout, and its weights are the operand of the second product as they come: lane
// half h has tokens 16 s + 8 u + 4 h + 0..3 (u = 0, 1) of the first, and the V tile lies in LDS in that order, [channel][step s][h][u].
// The softmax is one pass: reference of a row raised only when a score passes it by kLag (see kvlinc_rows.hip), one multiply-add, one
// exponential, half a maximum, half a sum and half a conversion a score.  Roundings to binary16: keys and values that are dequantized
// (codes times scales; a second term would double the products) and the weights; scores, sums and numerators stay binary32.
// The new rows come first, in their own basis; then the accumulators are rotated, and the cache's tiles follow.
#include <hip/hip_runtime.h>

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

constexpr int kTileWaves = 8, kTileThreads = 64 * kTileWaves, kTileRows = 32 * kTileWaves;
constexpr int kTileTokens = 64;
constexpr float kHeadroom = 8.0f, kLag = 5.0f;
constexpr float kFusedBound = 0x1p20f;  // references beyond it: the exponent is rounded as the reference is (see scores_to_weights)

typedef float float16_t __attribute__((ext_vector_type(16)));

// LDS tiles, 16-byte chunks permuted within a row so that neighbouring rows' reads, and the writers' pieces, fall on different banks.
// Keys: [64 tokens][16 chunks of 8 channels]; values: [128 channels][8 chunks of 8 tokens].
struct Tiles {
  u32x4_t k[kTileTokens][16];
  u32x4_t v[kHeadDim][8];
};
__device__ __forceinline__ int key_chunk(int t, int chunk) { return chunk ^ (t & 15); }
__device__ __forceinline__ int value_chunk(int ch, int chunk) { return chunk ^ (((ch >> 1) ^ (ch >> 4)) & 7); }
__device__ __forceinline__ void put_value_quad(Tiles& t, int ch, int quad, uint32_t a, uint32_t b) {  // tokens 4 quad .. 4 quad + 3
  const int chunk = 2 * (quad >> 2) + (quad & 1);
  reinterpret_cast<uint2*>(&t.v[ch][value_chunk(ch, chunk)])[(quad >> 1) & 1] = make_uint2(a, b);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ void barrier_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- tiles of raw rows [token][128] (new rows; keys of the window) -------------------------------------------------------------------
struct RawKeys {
  u32x4_t x[2];
};
__device__ __forceinline__ void load_raw_keys(RawKeys& r, const half_t* rows, int count, int tid) {
#pragma unroll
  for (int u = 0; u < 2; ++u) r.x[u] = reinterpret_cast<const u32x4_t*>(rows + (long long)min((tid >> 4) + 32 * u, count - 1) * kHeadDim)[tid & 15];
}
__device__ __forceinline__ void store_raw_keys(const RawKeys& r, Tiles& t, int tid) {
#pragma unroll
  for (int u = 0; u < 2; ++u) t.k[(tid >> 4) + 32 * u][key_chunk((tid >> 4) + 32 * u, tid & 15)] = r.x[u];
}
struct RawValues {
  u32x2_t x[4];  // 4 tokens (new rows) or 4 quads (window)
};
__device__ __forceinline__ void load_raw_values(RawValues& r, const half_t* rows, int count, int tid) {
#pragma unroll
  for (int u = 0; u < 4; ++u) r.x[u] = reinterpret_cast<const u32x2_t*>(rows + (long long)min(4 * (tid >> 5) + u, count - 1) * kHeadDim)[tid & 31];
}
__device__ __forceinline__ void store_raw_values(const RawValues& r, Tiles& t, int tid) {  // 4 tokens x 4 channels, turned over
  const int quad = tid >> 5, ch = 4 * (tid & 31);
  put_value_quad(t, ch, quad, low_halves(r.x[0].x, r.x[1].x), low_halves(r.x[2].x, r.x[3].x));
  put_value_quad(t, ch + 1, quad, high_halves(r.x[0].x, r.x[1].x), high_halves(r.x[2].x, r.x[3].x));
  put_value_quad(t, ch + 2, quad, low_halves(r.x[0].y, r.x[1].y), low_halves(r.x[2].y, r.x[3].y));
  put_value_quad(t, ch + 3, quad, high_halves(r.x[0].y, r.x[1].y), high_halves(r.x[2].y, r.x[3].y));
}
// the window's values, [slot / 4][channel][slot % 4]
__device__ __forceinline__ void load_window_values(RawValues& r, const half_t* v_win, int quad0, int quads, int tid) {
#pragma unroll
  for (int u = 0; u < 4; ++u)
    r.x[u] = reinterpret_cast<const u32x2_t*>(v_win)[min(quad0 + 4 * u + (tid >> 7), quads - 1) * kHeadDim + (tid & 127)];
}
__device__ __forceinline__ void store_window_values(const RawValues& r, Tiles& t, int tid) {
#pragma unroll
  for (int u = 0; u < 4; ++u) put_value_quad(t, tid & 127, 4 * u + (tid >> 7), r.x[u].x, r.x[u].y);
}

// ---- tiles of packed codes: one half (64 tokens) of a group -----------------------------------------------------------------------
template <int BITS>
struct Packed {
  uint32_t k[BITS / 2], v[2][BITS / 2];
  u32x4_t ks[2], kz[2];  // key scale and zero-point of the 16 channels of the key word
  u32x4_t sz[2][2];      // value (scale, zero-point) of tokens 16 i + 4 q4 + 2 hg + e, i = 4 half + 0..3: [hg][e]
};
// Thread: a key word (token 32 np + 16 nb + j of the half, channels 32 g + 16 w ..), and the two value words of channel 16 wave + j and the
// tokens 16 i + 4 q4 + 0..3.
template <int BITS>
__device__ __forceinline__ void load_packed(Packed<BITS>& p, const uint32_t* rec, int half, int tid) {
#pragma unroll
  for (int pl = 0; pl < BITS / 2; ++pl) p.k[pl] = rec[Rec<BITS>::kKeyTile + 1024 * pl + 512 * half + tid];
  const int at = 4 * ((tid >> 6) & 3) + 2 * (tid & 1);  // uint4 of the 16 channels' pairs
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    p.ks[i] = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyScale)[at + i];
    p.kz[i] = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyZero)[at + i];
  }
  const int n = tid >> 6, j = tid & 15, q4 = (tid >> 4) & 3;
#pragma unroll
  for (int hg = 0; hg < 2; ++hg) {
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl)
      p.v[hg][pl] = rec[Rec<BITS>::kValueTile + 1024 * pl + ((n >> 1) * 64 + j + 16 * ((q4 >> 1) + 2 * hg)) * 4 + 2 * (n & 1) + (q4 & 1)];
#pragma unroll
    for (int e = 0; e < 2; ++e) p.sz[hg][e] = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kValueSZ)[2 * (4 * q4 + 2 * hg + e) + half];
  }
}
// (code) s + z of two codes given as code - centre: one rounding; a sum beyond the largest binary16 number is that number.
template <int BITS>
__device__ __forceinline__ uint32_t dequantized(half2_t centred, uint32_t s, uint32_t z) {
  const half_t c = (half_t)Rec<BITS>::kCentre, top = (half_t)65504.0f;
  const half2_t v = __builtin_elementwise_fma(centred + half2_t{c, c}, as_h2(s), as_h2(z));
  return as_u32(__builtin_elementwise_min(v, half2_t{top, top}));
}
template <int BITS, int SEL>
__device__ __forceinline__ uint32_t key_pair(const uint32_t (&e)[BITS / 2], u32x4_t s, u32x4_t z) {
  return dequantized<BITS>(code_pair<BITS, SEL>(e, 1.0f), s[SEL], z[SEL]);
}
template <int BITS, int SEL>  // byte SEL of the value words: i = 2 SEL, 2 SEL + 1, at quads 4 i' + q4
__device__ __forceinline__ void value_quads(const Packed<BITS>& p, Tiles& t, int ch, int q4) {
  uint32_t lo[2], hi[2];
#pragma unroll
  for (int hg = 0; hg < 2; ++hg) {
    uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles n = nibbles_of(p.v[hg][pl]);
      e[pl] = n.first; o[pl] = n.second;
    }
    const uint32_t a = as_u32(code_pair<BITS, SEL>(e, 1.0f)), b = as_u32(code_pair<BITS, SEL>(o, 1.0f));
    const u32x4_t x = p.sz[hg][0], y = p.sz[hg][1];
    const uint32_t x0 = x[2 * (SEL & 1)], x1 = x[2 * (SEL & 1) + 1], y0 = y[2 * (SEL & 1)], y1 = y[2 * (SEL & 1) + 1];
    lo[hg] = dequantized<BITS>(as_h2(low_halves(a, b)), low_halves(x0, y0), high_halves(x0, y0));
    hi[hg] = dequantized<BITS>(as_h2(high_halves(a, b)), low_halves(x1, y1), high_halves(x1, y1));
  }
  const int i = 2 * (SEL & 1);
  put_value_quad(t, ch, 4 * i + q4, lo[0], lo[1]);
  put_value_quad(t, ch, 4 * (i + 1) + q4, hi[0], hi[1]);
}
template <int BITS>
__device__ __forceinline__ void store_packed(const Packed<BITS>& p, Tiles& t, int half, int tid) {
  const int u = tid >> 2, token = 32 * (u >> 6) + 16 * ((tid >> 1) & 1) + (u & 15), chunk = 4 * ((u >> 4) & 3) + 2 * (tid & 1);
  uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
  for (int pl = 0; pl < BITS / 2; ++pl) {
    const Nibbles n = nibbles_of(p.k[pl]);
    e[pl] = n.first; o[pl] = n.second;
  }
  t.k[token][key_chunk(token, chunk)] = u32x4_t{key_pair<BITS, 0>(e, p.ks[0], p.kz[0]), key_pair<BITS, 1>(e, p.ks[0], p.kz[0]),
                                                   key_pair<BITS, 2>(e, p.ks[0], p.kz[0]), key_pair<BITS, 3>(e, p.ks[0], p.kz[0])};
  t.k[token][key_chunk(token, chunk + 1)] = u32x4_t{key_pair<BITS, 0>(o, p.ks[1], p.kz[1]), key_pair<BITS, 1>(o, p.ks[1], p.kz[1]),
                                                       key_pair<BITS, 2>(o, p.ks[1], p.kz[1]), key_pair<BITS, 3>(o, p.ks[1], p.kz[1])};
  const int ch = 16 * (tid >> 6) + (tid & 15), q4 = (tid >> 4) & 3;
  if (half == 0) {
    value_quads<BITS, 0>(p, t, ch, q4);
    value_quads<BITS, 1>(p, t, ch, q4);
  } else {
    value_quads<BITS, 2>(p, t, ch, q4);
    value_quads<BITS, 3>(p, t, ch, q4);
  }
}
// Sliding values: the tokens of this half from slot `from` on take the window's values (written over the codes' by the thread that wrote them).
__device__ __forceinline__ void slide_values(Tiles& t, const half_t* v_win, int half, int from, int tid) {
  const int ch = 16 * (tid >> 6) + (tid & 15), q4 = (tid >> 4) & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int quad = 4 * i + q4, slot = kTileTokens * half + 4 * quad;
    if (slot + 3 < from) continue;
    const uint2 w = reinterpret_cast<const uint2*>(v_win)[(slot >> 2) * kHeadDim + ch];
    const int chunk = 2 * (quad >> 2) + (quad & 1);
    uint2* dst = reinterpret_cast<uint2*>(&t.v[ch][value_chunk(ch, chunk)]) + ((quad >> 1) & 1);
    const uint2 old = *dst;
    const uint32_t m0 = (slot >= from ? 0xffffu : 0u) | (slot + 1 >= from ? 0xffff0000u : 0u);
    const uint32_t m1 = (slot + 2 >= from ? 0xffffu : 0u) | (slot + 3 >= from ? 0xffff0000u : 0u);
    *dst = make_uint2((w.x & m0) | (old.x & ~m0), (w.y & m1) | (old.y & ~m1));
  }
}

// ---- a wave's rows ----------------------------------------------------------------------------------------------------------------
struct TileRows {
  half8_t q[8];      // channels 16 s + 8 h + 0..7 of this lane's row
  float m, l;        // reference (log2 domain), per-lane sum of the weights
  float16_t acc[4];  // numerator of channels 32 cb + 8 (r / 4) + 4 h + r % 4
};

__device__ __forceinline__ void raise_reference(TileRows& st, float largest) {  // largest score of this lane, log2 domain
  if (__builtin_amdgcn_ballot_w64(largest > st.m + (kHeadroom + kLag)) == 0) return;
  float x, y;
  pair_across<32>(largest, x, y);
  const float mx = fmaxf(x, y);
  const float to = mx > st.m + (kHeadroom + kLag) ? mx - kHeadroom : st.m;
  const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.m - to);
  st.m = to;
  st.l *= f;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb) st.acc[cb] *= f;
}

// One tile: 64 tokens, the first at position `at`.  masked: not every row sees all of them (p, low: of this lane's row).
__device__ __forceinline__ void attend_tile(TileRows& st, const Tiles& t, int at, int count, bool masked, int p, int low, int sinks, int lane) {
  const int i = lane & 31, h = lane >> 5;
  float16_t s[2];
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[tb][r] = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
      s[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(t.k[32 * tb + i][key_chunk(i, 2 * k + h)]), st.q[k], s[tb], 0, 0, 0);
  if (masked) {
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int tok = 32 * tb + 8 * (r >> 2) + 4 * h + (r & 3), pos = at + tok;
        if (!(tok < count && pos <= p && (pos >= low || pos < sinks))) s[tb][r] = -INFINITY;
      }
  }
  float mx = s[0][0];
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[tb][r]);
  raise_reference(st, mx * kLog2eSqrtD);
  const float m = st.m == -INFINITY ? 0.0f : st.m;
  if (__builtin_amdgcn_ballot_w64(fabsf(m) > kFusedBound) != 0) {
#pragma clang fp contract(off)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[tb][r] = __builtin_amdgcn_exp2f(s[tb][r] * kLog2eSqrtD - m);
  } else {
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[tb][r] = __builtin_amdgcn_exp2f(fmaf(s[tb][r], kLog2eSqrtD, -m));
  }
  half8_t P[4];
  const half2_t ones = {(half_t)1.0f, (half_t)1.0f};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    half2_t w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 8 * (k & 1) + 2 * u;
      w[u] = pack_h2(s[k >> 1][r], s[k >> 1][r + 1]);
      st.l = __builtin_amdgcn_fdot2(w[u], ones, st.l, false);
    }
    P[k] = as_h8(w[0], w[1], w[2], w[3]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) {
      const int ch = 32 * cb + i;
      st.acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_h8(t.v[ch][value_chunk(ch, 2 * k + h)]), P[k], st.acc[cb], 0, 0, 0);
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

// Grid, one-dimensional: see tile_unit.
template <int BITS, bool SLIDING>
__global__ __launch_bounds__(kTileThreads, 2) void tile_kernel(ContextCall a, int blocks) {
  __shared__ __align__(16) Tiles tiles[2];
  const kvlinc_cache& c = a.cache;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
  // Work items: split fastest, then (sequence, KV head), blocks of rows from the last (the longest) to the first.  Workgroups are dealt to
  // the 8 XCDs in turn: where the pairs divide by 8, those of one pair are 8 apart, so that its tiles come from one L2.
  const int pairs = c.B * c.H_kv;
  int id = blockIdx.x, split, bh, block;
  if (pairs % 8 == 0) {
    const int x = id & 7, y = id >> 3, per = pairs / 8;
    const int rest = y / a.splits;
    split = y - rest * a.splits;
    block = rest / per;
    bh = (rest - block * per) * 8 + x;
  } else {
    const int rest = id / a.splits;
    split = id - rest * a.splits;
    block = rest / pairs;
    bh = rest - block * pairs;
  }
  block = blocks - 1 - block;
  const int b = bh / c.H_kv, kvh = bh - b * c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int T = a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T;
  const int rows = T * gq, row0 = block * kTileRows;
  if (row0 >= rows) return;
  const int total = len.total();
  const long long head0 = (long long)b * c.H_q + (long long)kvh * gq;

  const int wave_row = row0 + 32 * wave, row = min(wave_row + (lane & 31), rows - 1);
  const bool idle = wave_row >= rows;
  const int my_i = row / gq, my_h = row - my_i * gq;
  const long long place = (head0 + my_h) * a.T + my_i;
  const int p = total + my_i, low = window_low(p, a.window);
  // of the wave's rows: positions p_first .. p_last, the first token of the first row's window, and of the last row's
  const int p_first = __builtin_amdgcn_readfirstlane(total + min(wave_row, rows - 1) / gq), p_last = __builtin_amdgcn_readfirstlane(total + min(wave_row + 31, rows - 1) / gq);
  const int low_first = window_low(p_first, a.window), low_last = window_low(p_last, a.window);

  TileRows st;
  {
    const uint4* src = reinterpret_cast<const uint4*>(a.q + place * kHeadDim) + h;
#pragma unroll
    for (int k = 0; k < 8; ++k) st.q[k] = as_h8(src[2 * k]);
  }
  st.m = -INFINITY;
  st.l = 0.0f;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.acc[cb][r] = 0.0f;

  // Tiles that some row of the block sees: of the new rows, of the window, halves of groups; this split has first .. last - 1 of them.
  const int last_i = min(row0 + kTileRows - 1, rows - 1) / gq, low_block = window_low(total + row0 / gq, a.window);
  const int new_from = a.sinks > total ? 0 : max(low_block - total, 0) / kTileTokens;
  const int n_new = last_i / kTileTokens + 1 - new_from;
  const int win_from = a.sinks > len.nq ? 0 : min(max(low_block - len.nq, 0), len.nr) / kTileTokens;
  const int n_win = (len.nr + kTileTokens - 1) / kTileTokens - win_from;
  const int halves = (len.nq + kTileTokens - 1) / kTileTokens, half_low = min(low_block / kTileTokens, halves);
  const int n_sink = a.window > 0 ? min((int)(((long long)a.sinks + kTileTokens - 1) / kTileTokens), half_low) : 0;
  const int n_tiles = n_new + n_win + halves - half_low + n_sink;
  const int first = (int)((long long)n_tiles * split / a.splits), last = (int)((long long)n_tiles * (split + 1) / a.splits);

  auto attend = [&](const Tiles& t, int at, int count) __attribute__((always_inline)) {
    if (idle || at > p_last || (at + count <= low_first && at >= a.sinks)) return;
    const bool masked = count < kTileTokens || at + kTileTokens - 1 > p_first || (at < low_last && at + kTileTokens > a.sinks);
    attend_tile(st, t, at, count, masked, p, low, a.sinks, lane);
  };

  const half_t* new_keys = a.k_new + (long long)bh * a.T * kHeadDim;
  const half_t* new_values = a.v_new + (long long)bh * a.T * kHeadDim;
  const half_t* k_win = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
  const half_t* v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
  auto half_of = [&](int item) { return item < n_sink ? item : item - n_sink + half_low; };

  // ---- raw tiles: the new rows, then the window ----
  const int raw_end = min(last, n_new + n_win);
  int item = first, buffer = 0;
  bool rotated = first >= n_new;
  if (item < raw_end) {
    RawKeys rk;
    RawValues rv;
    auto request = [&](int it) __attribute__((always_inline)) {
      const bool fresh = it < n_new;
      const int t0 = (fresh ? new_from + it : win_from + it - n_new) * kTileTokens;
      load_raw_keys(rk, (fresh ? new_keys : k_win) + (long long)t0 * kHeadDim, (fresh ? T : len.nr) - t0, tid);
      if (fresh) load_raw_values(rv, new_values + (long long)t0 * kHeadDim, T - t0, tid);
      else load_window_values(rv, v_win, t0 / 4, c.R / 4, tid);
    };
    auto put = [&](int it, Tiles& t) __attribute__((always_inline)) {
      store_raw_keys(rk, t, tid);
      if (it < n_new) store_raw_values(rv, t, tid);
      else store_window_values(rv, t, tid);
    };
    request(item);
    put(item, tiles[0]);
    barrier_lds();
    for (; item < raw_end; ++item) {
      const bool more = item + 1 < raw_end;
      if (more) request(item + 1);
      if (item == n_new) {
        rotate_tile_rows(st, lane);
        rotated = true;
      }
      const int t0 = item < n_new ? (new_from + item) * kTileTokens : (win_from + item - n_new) * kTileTokens;
      attend(tiles[buffer], (item < n_new ? total : len.nq) + t0, min((item < n_new ? T : len.nr) - t0, kTileTokens));
      buffer ^= 1;
      if (more) put(item + 1, tiles[buffer]);
      barrier_lds();
    }
  }
  // ---- halves of groups ----
  // (partial results of splits are in the cache's basis; a sequence without a cache that is not split stays in the new rows')
  const bool in_cache_basis = total > 0 || a.splits > 1;
  if (in_cache_basis && !rotated) rotate_tile_rows(st, lane);
  if (item < last) {
    const int skip = n_new + n_win;
    const int newest = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup ? len.groups() - 1 : -1;
    Packed<BITS> pk;
    auto request = [&](int it) __attribute__((always_inline)) {
      const int hf = half_of(it - skip);
      load_packed<BITS>(pk, rec0 + (long long)(hf >> 1) * Rec<BITS>::kWords, hf & 1, tid);
    };
    auto put = [&](int it, Tiles& t) __attribute__((always_inline)) {
      const int hf = half_of(it - skip);
      store_packed<BITS>(pk, t, hf & 1, tid);
      if (SLIDING && (hf >> 1) == newest) slide_values(t, v_win, hf & 1, len.nr, tid);
    };
    request(item);
    put(item, tiles[buffer]);
    barrier_lds();
    for (; item < last; ++item) {
      const bool more = item + 1 < last;
      if (more) request(item + 1);
      const int at = half_of(item - skip) * kTileTokens;
      attend(tiles[buffer], at, min(len.nq - at, kTileTokens));
      buffer ^= 1;
      if (more) put(item + 1, tiles[buffer]);
      barrier_lds();
    }
  }

  // ---- results ----
  if (idle) return;
  {
    float x, y;
    pair_across<32>(st.l, x, y);
    st.l = x + y;
  }
  const bool mine = wave_row + (lane & 31) < rows;
  if (a.splits > 1) {
    if (!mine) return;
    float* dst = a.part + (place * a.splits + split) * kPartStride;
    if (h == 0) { dst[0] = st.m; dst[1] = st.l; }
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(dst + 4 + 32 * cb + 2 * r + 4 * h) = make_float4(st.acc[cb][r], st.acc[cb][r + 1], st.acc[cb][r + 2], st.acc[cb][r + 3]);
    return;
  }
  if (a.corr != nullptr) {  // {C_d, -, -, -, C_n[128]}, as e^0 terms: both sides relative to max(m, 0)
    const float* corr = a.corr + place * kPartStride;
    const float to = fmaxf(st.m, 0.0f), f = __builtin_amdgcn_exp2f(st.m - to), w = __builtin_amdgcn_exp2f(-to);
    st.l = fmaf(w, corr[0], st.l * f);
#pragma unroll
    for (int cb = 0; cb < 4; ++cb)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 v = *reinterpret_cast<const float4*>(corr + 4 + 32 * cb + 2 * r + 4 * h);
        st.acc[cb][r] = fmaf(w, v.x, st.acc[cb][r] * f);
        st.acc[cb][r + 1] = fmaf(w, v.y, st.acc[cb][r + 1] * f);
        st.acc[cb][r + 2] = fmaf(w, v.z, st.acc[cb][r + 2] * f);
        st.acc[cb][r + 3] = fmaf(w, v.w, st.acc[cb][r + 3] * f);
      }
  }
  if (in_cache_basis) rotate_tile_rows(st, lane);
  if (!mine) return;
  const float inv = 1.0f / st.l;
  half_t* dst = a.out + place * kHeadDim;
#pragma unroll
  for (int cb = 0; cb < 4; ++cb)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<uint2*>(dst + 32 * cb + 2 * r + 4 * h) =
          make_uint2(as_u32(pack_h2(st.acc[cb][r] * inv, st.acc[cb][r + 1] * inv)), as_u32(pack_h2(st.acc[cb][r + 2] * inv, st.acc[cb][r + 3] * inv)));
}

}  // namespace

int launch_tiles(const ContextCall& a, hipStream_t stream) {
  const int blocks = (int)(((long long)a.T * a.gq + kTileRows - 1) / kTileRows);
  const dim3 grid((unsigned)((long long)blocks * a.cache.B * a.cache.H_kv * a.splits));
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  void (*kernel)(ContextCall, int) = a.cache.bits == 2 ? (sliding ? tile_kernel<2, true> : tile_kernel<2, false>) : (sliding ? tile_kernel<4, true> : tile_kernel<4, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), 0, stream, a, blocks);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  return a.splits > 1 ? launch_join(a, true, stream) : KVLINC_OK;
}

}  // namespace kvlinc
