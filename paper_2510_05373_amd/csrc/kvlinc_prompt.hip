// Prompt attention of many rows: blocks of 256 query rows over tiles of 64 tokens that the whole workgroup shares through LDS.
//
// Rows of a (sequence, KV head) are (token i, head h) pairs, row = i gq + h, so that a block covers few tokens and all heads share the
// tiles and the causal border.  Eight waves have 32 rows each; a tile is fetched into registers, turned into binary16 (packed codes: once
// for the 256 rows) and put into LDS.
//
// Both products run on v_mfma_f32_32x32x16_f16, transposed: S^T = K Q^T (rows = tokens, columns = query rows) and O^T = V^T P^T (rows =
// channels), so that a lane holds one query row throughout, and its weights are the operand of the second product as they come: lane
// half h has tokens 16 s + 8 u + 4 h + 0..3 (u = 0, 1) of the first, and the V tile lies in LDS in that order, [channel][step s][h][u].
// The softmax is one pass: reference of a row raised only when a score passes it by kHeadroom + kLag, one multiply-add, one
// exponential, half a maximum, half a sum and half a conversion a score.  Roundings to binary16: dequantized values (2^-12 of each; a second term
// would be 16 products a tile more), the weights, and dequantized keys, whose loss is added back in FP4 (see LowTile); scores, sums and numerators
// stay binary32.
// The new rows come first, in their own basis; then the accumulators are rotated, and the cache's tiles follow.
//
// Bound: vector instructions, softmax and unpacking: 128 tokens of 4 heads over 32k cached ones 137 to 144 us by the card (0.5 PFLOP/s), 64 tokens 90.
//
// Schedule.  A wave's tile is a matrix phase (P V of the tile, K Q of the next) and a vector phase (softmax, its share of a later tile into
// LDS), about as long as each other.  The two waves of a SIMD take them in turn: waves 4..7 run one phase behind waves 0..3, with a barrier
// at every change.
#include <hip/hip_runtime.h>

#include "kvlinc_tiles.h"

namespace kvlinc {
namespace {

// LDS tiles, 16-byte chunks permuted within a row so that neighbouring rows' reads, and the writers' pieces, fall on different banks.
// Keys: [64 tokens][16 chunks of 8 channels]; values: [128 channels][8 chunks of 8 tokens].
// A value tile is read one phase longer than a key tile: three of them.  Scales and zero-points of a group, 1 KB: one copy for each wave.
struct Tiles {
  u32x4_t k[2][kTileTokens][16];
  u32x4_t v[3][kHeadDim][8];
  u32x4_t meta[kTileWaves][64];
  LowTile low[2];  // as the key tiles
  // a wave's LowQuery (in registers all the time it made others spill, in every tile)
  u32x4_t q_low[kTileWaves][2][64];
  u32x4_t q_low_end[kTileWaves][64];
  // new rows whose values are not finite, as the value tiles: bits 0..3 of byte i are tokens 4 i .. 4 i + 3
  u32x4_t bad[3];
};
typedef u32x4_t (*KeyTile)[16];
typedef u32x4_t (*ValueTile)[8];
__device__ __forceinline__ int key_chunk(int t, int chunk) { return chunk ^ (t & 15); }
__device__ __forceinline__ int value_chunk(int ch, int chunk) { return chunk ^ (((ch >> 1) ^ (ch >> 4)) & 7); }
__device__ __forceinline__ void put_value_quad(ValueTile v, int ch, int quad, uint32_t a, uint32_t b) {  // tokens 4 quad .. 4 quad + 3
  const int chunk = 2 * (quad >> 2) + (quad & 1);
  reinterpret_cast<uint2*>(&v[ch][value_chunk(ch, chunk)])[(quad >> 1) & 1] = make_uint2(a, b);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// A thread's share of a tile on its way from memory to LDS.
//   raw rows [token][128] (new rows; keys of the window): x[0], x[1] = 8 channels of two tokens; values x[2], x[3] = 4 channels of 4 tokens,
//     or 4 tokens of a channel four times (the window's values, [slot / 4][channel][slot % 4]);
//   half a group of packed codes: x[0] 16 bytes of the record's scales and zero-points, which go through the wave's copy in LDS (held by the
//     threads that need them they take 32 registers); x[1], x[2] the key word (token 32 np + 16 nb + j of the half, channels 32 g + 16 w ..)
//     and the value words of channel 16 wave + j and the tokens 16 i + 4 q4 + 2 hg + 0, 1 of each plane.
template <int BITS>
struct Share {
  u32x4_t x[4];
};

template <int BITS>
__device__ __forceinline__ void load_raw_keys(Share<BITS>& s, const half_t* rows, int count, int tid) {
  asm("" : "+v"(tid));
#pragma unroll
  for (int u = 0; u < 2; ++u) s.x[u] = reinterpret_cast<const u32x4_t*>(rows + (long long)min((tid >> 4) + 32 * u, count - 1) * kHeadDim)[tid & 15];
}
template <int BITS>
__device__ __forceinline__ void store_raw_keys(const Share<BITS>& s, KeyTile t, int tid) {
  asm("" : "+v"(tid));
#pragma unroll
  for (int u = 0; u < 2; ++u) t[(tid >> 4) + 32 * u][key_chunk((tid >> 4) + 32 * u, tid & 15)] = s.x[u];
}
template <int BITS>
__device__ __forceinline__ void load_raw_values(Share<BITS>& s, const half_t* rows, int count, int tid) {
  asm("" : "+v"(tid));
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const u32x2_t w = reinterpret_cast<const u32x2_t*>(rows + (long long)min(4 * (tid >> 5) + u, count - 1) * kHeadDim)[tid & 31];
    s.x[2 + (u >> 1)][2 * (u & 1)] = w[0];
    s.x[2 + (u >> 1)][2 * (u & 1) + 1] = w[1];
  }
}
// 4 tokens x 4 channels, turned over.  What is not finite becomes 0, and its token is noted (see spoil_rows): 0.4 us of
// 100 tokens over an empty cache, 1 % of longer calls.
template <int BITS>
__device__ __forceinline__ void store_raw_values(Share<BITS>& s, ValueTile t, u32x4_t& bad, int tid) {
  asm("" : "+v"(tid));
  const int quad = tid >> 5, ch = 4 * (tid & 31);
  uint32_t here = 0, tokens = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) here |= not_finite(s.x[2][u]) | not_finite(s.x[3][u]);
  if (__builtin_amdgcn_ballot_w64(here != 0) != 0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {  // (32 lanes have the channels of the same tokens)
      const uint32_t a = s.x[2 + (u >> 1)][2 * (u & 1)], b = s.x[2 + (u >> 1)][2 * (u & 1) + 1];
      const uint64_t lanes = __builtin_amdgcn_ballot_w64((not_finite(a) | not_finite(b)) != 0);
      tokens |= (uint32_t)((tid & 32) != 0 ? lanes >> 32 : lanes & 0xffffffffu) != 0 ? 1u << u : 0u;
      s.x[2 + (u >> 1)][2 * (u & 1)] = finite_or_zero(a);
      s.x[2 + (u >> 1)][2 * (u & 1) + 1] = finite_or_zero(b);
    }
  }
  if ((tid & 31) == 0) reinterpret_cast<uint8_t*>(&bad)[quad] = (uint8_t)tokens;
  put_value_quad(t, ch, quad, low_halves(s.x[2][0], s.x[2][2]), low_halves(s.x[3][0], s.x[3][2]));
  put_value_quad(t, ch + 1, quad, high_halves(s.x[2][0], s.x[2][2]), high_halves(s.x[3][0], s.x[3][2]));
  put_value_quad(t, ch + 2, quad, low_halves(s.x[2][1], s.x[2][3]), low_halves(s.x[3][1], s.x[3][3]));
  put_value_quad(t, ch + 3, quad, high_halves(s.x[2][1], s.x[2][3]), high_halves(s.x[3][1], s.x[3][3]));
}
template <int BITS>
__device__ __forceinline__ void load_window_values(Share<BITS>& s, const half_t* v_win, int quad0, int quads, int tid) {
  asm("" : "+v"(tid));
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const u32x2_t w = reinterpret_cast<const u32x2_t*>(v_win)[min(quad0 + 4 * u + (tid >> 7), quads - 1) * kHeadDim + (tid & 127)];
    s.x[2 + (u >> 1)][2 * (u & 1)] = w[0];
    s.x[2 + (u >> 1)][2 * (u & 1) + 1] = w[1];
  }
}
template <int BITS>
__device__ __forceinline__ void store_window_values(const Share<BITS>& s, ValueTile t, int tid) {
  asm("" : "+v"(tid));
#pragma unroll
  for (int u = 0; u < 4; ++u) put_value_quad(t, tid & 127, 4 * u + (tid >> 7), s.x[2 + (u >> 1)][2 * (u & 1)], s.x[2 + (u >> 1)][2 * (u & 1) + 1]);
}

template <int BITS>
__device__ __forceinline__ void load_packed(Share<BITS>& s, const uint32_t* rec, int half, int tid) {
  asm("" : "+v"(tid));
  const int n = tid >> 6, j = tid & 15, q4 = (tid >> 4) & 3;
  s.x[0] = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyScale)[tid & 63];
#pragma unroll
  for (int pl = 0; pl < BITS / 2; ++pl) {
    s.x[1 + pl][0] = rec[Rec<BITS>::kKeyTile + 1024 * pl + 512 * half + tid];
#pragma unroll
    for (int hg = 0; hg < 2; ++hg)
      s.x[1 + pl][1 + hg] = rec[Rec<BITS>::kValueTile + 1024 * pl + ((n >> 1) * 64 + j + 16 * ((q4 >> 1) + 2 * hg)) * 4 + 2 * (n & 1) + (q4 & 1)];
  }
}
static_assert(Rec<2>::kKeyZero == Rec<2>::kKeyScale + 64 && Rec<2>::kValueSZ == Rec<2>::kKeyScale + 128 && Rec<2>::kWords == Rec<2>::kKeyScale + 256, "256 words");
// (code) s + z of two codes given as code - centre, one rounding; a sum beyond the largest binary16 number (the quantizer's scale was rounded
// up) is that number.
template <int BITS>
__device__ __forceinline__ uint32_t dequantized(half2_t centred, uint32_t s, uint32_t z) {
  const half_t c = (half_t)Rec<BITS>::kCentre, top = (half_t)65504.0f;
  return as_u32(__builtin_elementwise_min(__builtin_elementwise_fma(centred + half2_t{c, c}, as_h2(s), as_h2(z)), half2_t{top, top}));
}
// Channels 2 SEL, 2 SEL + 1 of eight, and what their rounding leaves.
template <int BITS, int SEL>
__device__ __forceinline__ uint32_t key_pair(const uint32_t (&e)[BITS / 2], u32x4_t s, u32x4_t z, float (&rest)[8]) {
  const half2_t centred = code_pair<BITS, SEL>(e, 1.0f), ss = as_h2(s[SEL]), zz = as_h2(z[SEL]);
  const uint32_t key = dequantized<BITS>(centred, s[SEL], z[SEL]);
  const half_t c = (half_t)Rec<BITS>::kCentre;
  const half2_t code = centred + half2_t{c, c};
#pragma unroll
  for (int i = 0; i < 2; ++i) rest[2 * SEL + i] = fmaf((float)code[i], (float)ss[i], (float)zz[i]) - (float)as_h2(key)[i];
  return key;
}
template <int BITS>
__device__ __forceinline__ u32x4_t key_chunk_of(const uint32_t (&e)[BITS / 2], u32x4_t s, u32x4_t z, float (&rest)[8]) {
  return u32x4_t{key_pair<BITS, 0>(e, s, z, rest), key_pair<BITS, 1>(e, s, z, rest), key_pair<BITS, 2>(e, s, z, rest), key_pair<BITS, 3>(e, s, z, rest)};
}
// Tokens i' = 2 SEL, 2 SEL + 1 of a half (quads 4 i' + q4) from byte SEL of the value words.
template <int BITS, int SEL>
__device__ __forceinline__ void value_quads(const uint32_t (&e)[2][BITS / 2], const uint32_t (&o)[2][BITS / 2], const u32x4_t (&sz)[4], ValueTile t, int ch, int q4) {
  uint32_t lo[2], hi[2];
#pragma unroll
  for (int hg = 0; hg < 2; ++hg) {
    const uint32_t a = as_u32(code_pair<BITS, SEL>(e[hg], 1.0f)), b = as_u32(code_pair<BITS, SEL>(o[hg], 1.0f));
    const u32x4_t x = sz[2 * hg], y = sz[2 * hg + 1];
    lo[hg] = dequantized<BITS>(as_h2(low_halves(a, b)), low_halves(x[2 * SEL], y[2 * SEL]), high_halves(x[2 * SEL], y[2 * SEL]));
    hi[hg] = dequantized<BITS>(as_h2(high_halves(a, b)), low_halves(x[2 * SEL + 1], y[2 * SEL + 1]), high_halves(x[2 * SEL + 1], y[2 * SEL + 1]));
  }
  put_value_quad(t, ch, 8 * SEL + q4, lo[0], lo[1]);
  put_value_quad(t, ch, 8 * SEL + 4 + q4, hi[0], hi[1]);
}
template <int BITS>
__device__ __forceinline__ void store_packed(const Share<BITS>& s, u32x4_t* meta, KeyTile kt, LowTile& low, ValueTile vt, int half, int tid) {
  asm("" : "+v"(tid));  // (addresses formed here, not kept over the loop)
  meta[tid & 63] = s.x[0];
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS instructions stay in order)
  {
    const int u = tid >> 2, token = 32 * (u >> 6) + 16 * ((tid >> 1) & 1) + (u & 15), chunk = 4 * ((u >> 4) & 3) + 2 * (tid & 1);
    uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles n = nibbles_of(s.x[1 + pl][0]);
      e[pl] = n.first; o[pl] = n.second;
    }
    const u32x4_t s0 = meta[chunk], s1 = meta[chunk + 1], z0 = meta[16 + chunk], z1 = meta[17 + chunk];  // a chunk of 8 channels is 16 bytes here, too
    float r0[8], r1[8];
    const u32x4_t k0 = key_chunk_of<BITS>(e, s0, z0, r0), k1 = key_chunk_of<BITS>(o, s1, z1, r1);
    kt[token][key_chunk(token, chunk)] = k0;
    kt[token][key_chunk(token, chunk + 1)] = k1;
    // the largest of the token's 32 channels: this thread's 16 and its neighbour's (as integers, halves apart)
    uint32_t even = 0, odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      even = max(even, max(k0[i] & 0x7fffu, k1[i] & 0x7fffu));
      odd = max(odd, max(k0[i] & 0x7fff0000u, k1[i] & 0x7fff0000u));
    }
    uint32_t top = max(even, odd >> 16);
    top = max(top, dpp_u<kQuadSwap1>(top));
    const uint32_t scale = low_scale_of(top);
    const float by = bits_f32(scale << 23);
    const int g = chunk >> 2;
    reinterpret_cast<u32x2_t*>(&low.k[token][low_chunk(token, g)])[tid & 1] = u32x2_t{fp4_of(r0, by), fp4_of(r1, by)};
    if ((tid & 1) == 0) reinterpret_cast<uint8_t*>(&low.scale[token])[g] = (uint8_t)scale;
  }
  __builtin_amdgcn_sched_barrier(0);
  const int ch = 16 * (tid >> 6) + (tid & 15), q4 = (tid >> 4) & 3;
  // word 8 t + n of the value pairs is token 16 n + t: tokens 16 i + 4 q4 + 2 hg + e, i = 4 half + 0..3, in 16 bytes
  const u32x4_t sz[4] = {meta[32 + 2 * (4 * q4) + half], meta[32 + 2 * (4 * q4 + 1) + half], meta[32 + 2 * (4 * q4 + 2) + half], meta[32 + 2 * (4 * q4 + 3) + half]};
  uint32_t e[2][BITS / 2], o[2][BITS / 2];
#pragma unroll
  for (int hg = 0; hg < 2; ++hg)
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles n = nibbles_of(s.x[1 + pl][1 + hg] >> (16 * half));  // (bytes 2 half, 2 half + 1 of a value word are these tokens)
      e[hg][pl] = n.first; o[hg][pl] = n.second;
    }
  value_quads<BITS, 0>(e, o, sz, vt, ch, q4);
  value_quads<BITS, 1>(e, o, sz, vt, ch, q4);
}
// Sliding values: the tokens of this half from slot `from` on take the window's values (written over the codes' by the thread that wrote them).
__device__ __forceinline__ void slide_values(ValueTile t, const half_t* v_win, int half, int from, int tid) {
  const int ch = 16 * (tid >> 6) + (tid & 15), q4 = (tid >> 4) & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int quad = 4 * i + q4, slot = kTileTokens * half + 4 * quad;
    if (slot + 3 < from) continue;
    const uint2 w = reinterpret_cast<const uint2*>(v_win)[(slot >> 2) * kHeadDim + ch];
    const int chunk = 2 * (quad >> 2) + (quad & 1);
    uint2* dst = reinterpret_cast<uint2*>(&t[ch][value_chunk(ch, chunk)]) + ((quad >> 1) & 1);
    const uint2 old = *dst;
    const uint32_t m0 = (slot >= from ? 0xffffu : 0u) | (slot + 1 >= from ? 0xffff0000u : 0u);
    const uint32_t m1 = (slot + 2 >= from ? 0xffffu : 0u) | (slot + 3 >= from ? 0xffff0000u : 0u);
    *dst = make_uint2((w.x & m0) | (old.x & ~m0), (w.y & m1) | (old.y & ~m1));
  }
}

// S^T = K Q^T of a tile.  A lane's chunks 2 k + h of rows i and 32 + i: key_chunk only flips address bits, so they are one address with
// k in bits 5..7 flipped (chunk and i & 15 are four bits).
__device__ __forceinline__ void tile_scores(TileRows& st, KeyTile t, int lane) {
  asm("" : "+v"(lane));
  const int i = lane & 31, base = i * 256 + 16 * key_chunk(i, lane >> 5);
#pragma unroll
  for (int tb = 0; tb < 2; ++tb)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.s[tb][r] = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) st.s[tb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_operand(t, (base ^ (32 * k)) + 8192 * tb), st.q[k], st.s[tb], 0, 0, 0);
}
// O^T += V^T P^T.  Chunks 2 k + h of rows 32 cb + i: the same, value_chunk of row 32 cb + i being that of row i with 2 cb flipped.
__device__ __forceinline__ void tile_values(TileRows& st, ValueTile t, int lane) {
  asm("" : "+v"(lane));
  const int i = lane & 31, base = i * 128 + 16 * value_chunk(i, lane >> 5);
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int cb = 0; cb < 4; ++cb) st.acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_operand(t, (base ^ (32 * (k ^ cb))) + 4096 * cb), st.p[k], st.acc[cb], 0, 0, 0);
}
// Grid, one-dimensional: see place_of_block.
template <int BITS, bool SLIDING>
__global__ __launch_bounds__(kTileThreads, 2) void tile_kernel(ContextCall a, int blocks) {
  __shared__ __align__(16) Tiles tiles;
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
  int low_scale = 0;
  start_rows(st, a.q + wr.place * kHeadDim, lane);
  if (len.nq > 0) {
    const LowQuery q = low_query(a.q + wr.place * kHeadDim, lane);
#pragma unroll
    for (int j = 0; j < 2; ++j) tiles.q_low[wave][j][lane] = u32x4_t{q.q[j][0], q.q[j][1], q.q[j][2], q.q[j][3]};
    tiles.q_low_end[wave][lane] = u32x4_t{q.q[0][4], q.q[0][5], q.q[1][4], q.q[1][5]};
    low_scale = q.scale;
  }
  auto add_low = [&](const LowTile& t) __attribute__((always_inline)) {
    int lane = tid & 63;
    asm("" : "+v"(lane));
    const u32x4_t a0 = tiles.q_low[wave][0][lane], a1 = tiles.q_low[wave][1][lane], e = tiles.q_low_end[wave][lane];
    LowQuery q;
    q.q[0] = u32x6_t{a0[0], a0[1], a0[2], a0[3], e[0], e[1]};
    q.q[1] = u32x6_t{a1[0], a1[1], a1[2], a1[3], e[2], e[3]};
    q.scale = low_scale;
    low_scores(st, t, q, lane);
  };

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

  const half_t* new_keys = a.k_new + (long long)bh * a.T * kHeadDim;
  const half_t* new_values = a.v_new + (long long)bh * a.T * kHeadDim;
  const half_t* k_win = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
  const half_t* v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
  const int raw = n_new + n_win, newest = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup ? len.groups() - 1 : -1;
  auto half_of = [&](int it) { return it - raw < n_sink ? it - raw : it - raw - n_sink + half_low; };

  Share<BITS> sh;
  auto request = [&](int it) __attribute__((always_inline)) {
    if (it < raw) {
      const bool fresh = it < n_new;
      const int t0 = (fresh ? new_from + it : win_from + it - n_new) * kTileTokens;
      load_raw_keys<BITS>(sh, (fresh ? new_keys : k_win) + (long long)t0 * kHeadDim, (fresh ? T : len.nr) - t0, tid);
      if (fresh) load_raw_values<BITS>(sh, new_values + (long long)t0 * kHeadDim, T - t0, tid);
      else load_window_values<BITS>(sh, v_win, t0 / 4, c.R / 4, tid);
    } else {
      const int hf = half_of(it);
      load_packed<BITS>(sh, rec0 + (long long)(hf >> 1) * Rec<BITS>::kWords, hf & 1, tid);
    }
  };
  auto put = [&](int it, int kb, int vb) __attribute__((always_inline)) {
    if (it < raw) {
      store_raw_keys<BITS>(sh, tiles.k[kb], tid);
      if (it < n_new) store_raw_values<BITS>(sh, tiles.v[vb], tiles.bad[vb], tid);
      else store_window_values<BITS>(sh, tiles.v[vb], tid);
    } else {
      const int hf = half_of(it);
      store_packed<BITS>(sh, tiles.meta[wave], tiles.k[kb], tiles.low[kb], tiles.v[vb], hf & 1, tid);
      if (SLIDING && (hf >> 1) == newest) slide_values(tiles.v[vb], v_win, hf & 1, len.nr, tid);
    }
  };

  // Tile `first` + k lies in key tile k % 2 and value tile k % 3.  Waves 0..3 put theirs one tile ahead of the softmax, waves 4..7, a phase
  // behind them, two: all of a tile is there when waves 0..3 take its keys, and what it is written over has been read by all.
  const int n = last - first, behind = wave >> 2;
  bool rotated = first >= n_new;
  if (n > 0) {
    int to = 0, kb_put = 0, vb_put = 0;  // the next tile to put, and where
    auto put_next = [&]() __attribute__((always_inline)) {
      put(first + to, kb_put, vb_put);
      ++to;
      kb_put ^= 1;
      vb_put = vb_put == 2 ? 0 : vb_put + 1;
      if (to < n) request(first + to);
    };
    request(first);
#pragma unroll 1
    for (int k = 0; k <= behind && to < n; ++k) put_next();
    next_phase();
    if (behind) next_phase();
    // q has arrived from here on: left to its first use in the loop, the wait there would be for a tile under way, too
#pragma unroll
    for (int k = 0; k < 8; ++k) asm volatile("" : "+v"(st.q[k]));
    if (!wr.idle) tile_scores(st, tiles.k[0], lane);
    if (!wr.idle && first >= raw) add_low(tiles.low[0]);
    next_phase();
    int vb = 0;
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      // vector phase
      const int item = first + k;
      if (item == n_new && !rotated) {
        rotate_tile_rows(st, lane);
        rotated = true;
      }
      int at, count;
      if (item < raw) {
        const int t0 = (item < n_new ? new_from + item : win_from + item - n_new) * kTileTokens;
        at = (item < n_new ? total : len.nq) + t0;
        count = min((item < n_new ? T : len.nr) - t0, kTileTokens);
      } else {
        at = half_of(item) * kTileTokens;
        count = min(len.nq - at, kTileTokens);
      }
      const bool live = wave_sees(wr, a, at, count);
      if (live) tile_weights(st, at, count, wave_masked(wr, a, at, count), wr.p, wr.low, a.sinks, lane);
      if (item < n_new) {
        const u32x4_t b = tiles.bad[vb];
        if (__builtin_amdgcn_readfirstlane(b[0] | b[1] | b[2] | b[3]) != 0) {
          uint64_t bad = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) bad |= (uint64_t)(b[i >> 2] >> (8 * (i & 3)) & 15u) << (4 * i);
          spoil_rows(st, bad, at, wr.p, wr.low, a.sinks);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (to < n) put_next();
      next_phase();
      // matrix phase
      if (live) {
        tile_values(st, tiles.v[vb], lane);
        tile_scores(st, tiles.k[(k + 1) & 1], lane);  // (of the last tile: what the other key tile held; not used)
        matrix_order<32>();
      } else if (!wr.idle) {
        tile_scores(st, tiles.k[(k + 1) & 1], lane);
        matrix_order<16>();
      }
      if (item + 1 >= raw && !wr.idle) add_low(tiles.low[(k + 1) & 1]);
      vb = vb == 2 ? 0 : vb + 1;
      next_phase();
    }
    if (!behind) next_phase();
  }
  // (partial results of splits are in the cache's basis; a sequence without a cache that is not split stays in the new rows')
  const bool in_cache_basis = total > 0 || a.splits > 1;
  if (in_cache_basis && !rotated) rotate_tile_rows(st, lane);
  store_results(st, a, wr, split, in_cache_basis, lane);
}

}  // namespace

int launch_tiles(const ContextCall& a, hipStream_t stream) {
  const int blocks = (int)(((long long)a.T * a.gq + kTileRows - 1) / kTileRows);
  const dim3 grid((unsigned)((long long)blocks * a.cache.B * a.cache.H_kv * a.splits));
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  void (*kernel)(ContextCall, int) = a.cache.bits == 2 ? (sliding ? tile_kernel<2, true> : tile_kernel<2, false>) : (sliding ? tile_kernel<4, true> : tile_kernel<4, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kTileThreads), 0, stream, a, blocks);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  return a.splits > 1 ? launch_join(a, stream) : KVLINC_OK;
}

}  // namespace kvlinc
