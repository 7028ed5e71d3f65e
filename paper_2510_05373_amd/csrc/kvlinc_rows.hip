// Attention of few query rows, or of one query a sequence behind a sliding window, read directly from the packed cache.
//
// Rows of a (sequence, KV head) are (token i, head h) pairs, row = i gq + h.  A wave takes blocks of tokens on its own, without a
// barrier: groups of 128 packed tokens, or 32 raw ones (the cache's window, the new rows), and keeps a running maximum, sum and numerator
// of its 16 NR rows; the workgroup's four waves are joined through LDS, the splits of a context through memory.
//
// Both products run on v_mfma_f32_16x16x32_f16, transposed: S^T = K Q^T (rows = tokens, columns = query rows) and
// O^T = V^T P^T (rows = channels, columns = query rows), so that a lane holds one query row, lane % 16, throughout, and the weights it
// forms are the operand it feeds.  For that the tokens of a block of 16 are taken in the order pi(4 g + r) = 8 (g % 2) + 2 (g / 2) +
// r % 2 + 4 (r / 2) (g = lane / 16): what a lane of the second product has of a value tile's words.
// Codes become binary16 numbers code - centre in one instruction a pair and stay unscaled: the key scales ride on the query
// (q s in two binary16 terms, the second what the first leaves: 2^-22 of it), the value scales on the weights.  With the scale on the
// tile instead, every group would cost 128 multiply-adds a lane and 16 rows, where this takes 32; the second term keeps the scores as
// exact as binary32 products of the scales would be.  Zero-points and centring are sums over channels resp. tokens.
// Weights are rounded to binary16 once, for the second product: 2^-12 of each at most, of no common sign.  They are kept near 2^8 (see
// kHeadroom), where the smallest that count are normal numbers; sums of weights are taken before the rounding, in binary32.
#include <hip/hip_runtime.h>

#include "kvlinc_codes.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

constexpr int kRowWaves = 4;
constexpr int kRawTokens = 32;
// The reference of a row is its largest score less kHeadroom when it is set, and is set anew when a score passes it by kHeadroom + kLag
// (most blocks only compare): weights stay below 2^13, and p s with s < 2 below binary16's largest number.
constexpr float kHeadroom = 8.0f, kLag = 5.0f;
constexpr float kFusedBound = 0x1p20f;

__device__ __forceinline__ int token_order(int i) { return 8 * ((i >> 2) & 1) + 2 * (i >> 3) + (i & 1) + 4 * ((i >> 1) & 1); }

template <int BITS>
struct Record {
  u32x4_t kw[2 * BITS];  // key words: kw[4 plane + m] = token blocks 2 m (x, y) and 2 m + 1 (z, w)
  u32x4_t vw[2 * BITS];  // value words: channel blocks 2 m and 2 m + 1
  u32x4_t meta;          // 16 bytes of the record's 1 KB of scales and zero-points
};
template <int BITS>
__device__ __forceinline__ void load_key_part(Record<BITS>& r, const uint32_t* rec, int lane) {
  const u32x4_t* kt = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyTile) + token_order(lane & 15) + (lane & 48);
#pragma unroll
  for (int m = 0; m < 2 * BITS; ++m) r.kw[m] = __builtin_nontemporal_load(kt + 64 * m);
  r.meta = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kKeyScale) + lane);
}
template <int BITS>
__device__ __forceinline__ void load_value_part(Record<BITS>& r, const uint32_t* rec, int lane) {
  const u32x4_t* vt = reinterpret_cast<const u32x4_t*>(rec + Rec<BITS>::kValueTile) + lane;
#pragma unroll
  for (int m = 0; m < 2 * BITS; ++m) r.vw[m] = __builtin_nontemporal_load(vt + 64 * m);
}
static_assert(Rec<2>::kKeyZero == Rec<2>::kKeyScale + 64 && Rec<2>::kValueSZ == Rec<2>::kKeyScale + 128 && Rec<2>::kWords == Rec<2>::kKeyScale + 256, "256 words");

// A wave's copy of a group's scales and zero-points in LDS: [0..15] key scales, [16..31] key zero-points, 8 channels each; [32 + 2 t + u]
// value (scale, zero-point) of tokens 16 (4 u + i) + t, i = 0..3.  The exponent of the group's largest value scale is taken out of them on
// the way (it goes to the codes, exactly: weight times scale then stays in binary16's range whatever the values' magnitude) and returned.
template <int BITS>
__device__ __forceinline__ int put_meta(const Record<BITS>& r, u32x4_t* meta, int lane) {
  uint32_t top = 0;  // scales are not negative: their bit patterns order like the numbers
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, r.meta[i] & 0xffffu);
  top = lane >= 32 ? top : 0u;
  top = max(top, dpp_u<kRowRor1>(top));
  top = max(top, dpp_u<kRowRor2>(top));
  top = max(top, dpp_u<kRowRor4>(top));
  top = max(top, dpp_u<kRowRor8>(top));
  const int e = (int)(max(max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)) >> 10, 3u)) - 15;  // -12 .. 15: the codes times 2^e are normal numbers
  const half2_t unscale = {(half_t)(lane >= 32 ? bits_f32((uint32_t)(127 - e) << 23) : 1.0f), (half_t)1.0f};
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = as_u32(as_h2(r.meta[i]) * unscale);
  meta[lane] = w;
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS instructions stay in order)
  return e;
}

template <int NR>
struct Rows {
  half8_t q[NR][4];       // query of this lane's row, channels 32 g + 8 step .. + 7, times 2^-e (largest magnitude in [1/2, 1))
  float unit[NR];         // 2^e log2(e) / sqrt(d)
  int p[NR], low[NR];     // position, first token of its window
  float m[NR];            // reference (the same in the four lanes of a row), log2 domain; -inf: nothing seen yet
  float l[NR], mid[NR];   // per-lane sums of the weights, and of weight times (zero-point + centre scale): the same for all channels
  float4_t acc[NR][8];    // numerator of channels 16 n + 4 g + 0..3
};

template <int NR>
__device__ __forceinline__ void set_reference(Rows<NR>& st, int k, float largest) {  // largest: of this lane's scores
  if (__builtin_amdgcn_ballot_w64(largest > st.m[k] + (kHeadroom + kLag)) == 0) return;
  float x, y;
  pair_across<16>(largest, x, y);
  pair_across<32>(fmaxf(x, y), x, y);
  const float mx = fmaxf(x, y);
  const float to = mx > st.m[k] + (kHeadroom + kLag) ? mx - kHeadroom : st.m[k];
  const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.m[k] - to);  // (0 where nothing was seen)
  st.m[k] = to;
  st.l[k] *= f;
  st.mid[k] *= f;
#pragma unroll
  for (int n = 0; n < 8; ++n) st.acc[k][n] *= f;
}
__device__ __forceinline__ float finite_reference(float m) { return m == -INFINITY ? 0.0f : m; }

// Token of register r, block n of the tile whose first token is `at`, or -1 beyond its `count` tokens; and whether a row sees it.
__device__ __forceinline__ bool seen(int t, int at, int count, int p, int low, int sinks) {
  const int pos = at + t;
  return t < count && pos <= p && (pos >= low || pos < sinks);
}

// O^T += V^T P^T with the window's fp16 values of 16-token blocks first .. first + 2 count - 1 (two a product), weights w[n][r] by block.
// v_res is [slot / 4][channel][slot % 4]: a lane takes two neighbouring slots at a time.
template <int NR, int NB>
__device__ __forceinline__ void window_values(Rows<NR>& st, const half_t* v_win, int quads, int first, const float (&w)[NR][NB][4], int lane) {
  const int g = lane >> 4, a = 8 * (g & 1) + 2 * (g >> 1);
#pragma unroll
  for (int s = 0; s < NB / 2; ++s) {
    half8_t P[NR];
#pragma unroll
    for (int k = 0; k < NR; ++k)
      P[k] = as_h8(pack_h2(w[k][2 * s][0], w[k][2 * s][1]), pack_h2(w[k][2 * s][2], w[k][2 * s][3]), pack_h2(w[k][2 * s + 1][0], w[k][2 * s + 1][1]),
                   pack_h2(w[k][2 * s + 1][2], w[k][2 * s + 1][3]));
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      uint32_t v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {  // (slots beyond the window take its last quad's: their weights are 0 and the window is finite)
        const int slot = 16 * (first + 2 * s + (u >> 1)) + a + 4 * (u & 1);
        v[u] = *reinterpret_cast<const uint32_t*>(v_win + ((long long)min(slot >> 2, quads - 1) * kHeadDim + 16 * n + (lane & 15)) * 4 + (slot & 3));
      }
      const half8_t V = as_h8(make_uint4(v[0], v[1], v[2], v[3]));
#pragma unroll
      for (int k = 0; k < NR; ++k) st.acc[k][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(V, P[k], st.acc[k][n], 0, 0, 0);
    }
    asm volatile("" ::: "memory");  // (the next blocks' loads stay behind these products: all at once they spilled)
  }
}

// One group of 128 packed tokens, the first at position `at`, `count` of them there.  masked: some row does not see all of them.
// SLIDING: tokens from fp16_from on take their values from the window.
template <int BITS, int NR>
__device__ __forceinline__ void group_scores(Rows<NR>& st, const Record<BITS>& rec, const u32x4_t* meta, int at, int count, bool masked, int sinks,
                                             int lane, float (&x)[NR][8][4], float (&base)[NR]) {
  half8_t hi[NR][4], lo[NR][4];
  float bias[NR];
  {
    float bz[NR], bs[NR];
#pragma unroll
    for (int k = 0; k < NR; ++k) bz[k] = bs[k] = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4_t S = meta[4 * (lane >> 4) + s], Z = meta[16 + 4 * (lane >> 4) + s];
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        const u32x4_t qq = __builtin_bit_cast(u32x4_t, st.q[k][s]);
        u32x4_t h, r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const half2_t a = as_h2(qq[i]), sc = as_h2(S[i]);
          const half2_t t = a * sc;
          h[i] = as_u32(t);
          r[i] = as_u32(__builtin_elementwise_fma(a, sc, -t));
          bz[k] = __builtin_amdgcn_fdot2(a, as_h2(Z[i]), bz[k], false);
          bs[k] = __builtin_amdgcn_fdot2(a, sc, bs[k], false);
        }
        hi[k][s] = as_h8(h);
        lo[k][s] = as_h8(r);
      }
    }
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      float a, b;
      pair_across<16>(fmaf(bs[k], Rec<BITS>::kCentre, bz[k]), a, b);
      pair_across<32>(a + b, a, b);
      bias[k] = (a + b) * st.unit[k];
    }
  }
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      half8_t A[4];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
        for (int pl = 0; pl < BITS / 2; ++pl) {
          const Nibbles nb = nibbles_of(rec.kw[4 * pl + m][2 * hf + w]);
          e[pl] = nb.first; o[pl] = nb.second;
        }
        A[2 * w] = as_h8(code_pair<BITS, 0>(e, 1.0f), code_pair<BITS, 1>(e, 1.0f), code_pair<BITS, 2>(e, 1.0f), code_pair<BITS, 3>(e, 1.0f));
        A[2 * w + 1] = as_h8(code_pair<BITS, 0>(o, 1.0f), code_pair<BITS, 1>(o, 1.0f), code_pair<BITS, 2>(o, 1.0f), code_pair<BITS, 3>(o, 1.0f));
      }
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[s], lo[k][s], d, 0, 0, 0);
#pragma unroll
        for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[s], hi[k][s], d, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[k][2 * m + hf][r] = d[r];
      }
    }
  if (masked) {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const int end = min(count, st.p[k] - at + 1), from = st.low[k] - at, first = sinks - at;
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = 16 * n + token_order(4 * (lane >> 4) + r);
          x[k][n][r] = (t < end) & ((t >= from) | (t < first)) ? x[k][n][r] : -INFINITY;
        }
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    float mx = x[k][0][0];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[k][n][r]);
    set_reference<NR>(st, k, fmaf(mx, st.unit[k], bias[k]));
    const float m = finite_reference(st.m[k]);
    base[k] = bias[k] - m;
    // References and biases thousands beyond what ordinary keys and queries give: the exponents are rounded as the reference was (the
    // score itself, then its distance from the reference), or the exponent of the largest weight would be what the roundings leave.
    if (__builtin_amdgcn_ballot_w64(fmaxf(fabsf(m), fabsf(bias[k])) > kFusedBound) != 0) {
#pragma clang fp contract(off)
      const float back = 1.0f / st.unit[k];
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[k][n][r] = (__builtin_fmaf(x[k][n][r], st.unit[k], bias[k]) - m) * back;
      base[k] = 0.0f;
    }
  }
}

// Scores become weights; O^T += V^T P^T of the group.  e: see put_meta.
template <int BITS, int NR, bool SLIDING>
__device__ __forceinline__ void group_values(Rows<NR>& st, const Record<BITS>& rec, const u32x4_t* meta, int e, float (&x)[NR][8][4], const float (&base)[NR],
                                             int fp16_from, const half_t* v_win, int quads, int lane) {
  const float scale = bits_f32((uint32_t)(127 + e) << 23);
  half8_t P[NR][4];
  float l[NR], ys[NR], zs[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) l[k] = ys[k] = zs[k] = 0.0f;
  const half2_t ones = {(half_t)1.0f, (half_t)1.0f};
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = token_order(4 * (lane >> 4) + r);
    const u32x4_t z0 = meta[32 + 2 * t], z1 = meta[33 + 2 * t];
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        float y[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int n = 2 * s + u;
          const half2_t sz = as_h2(n < 4 ? z0[n] : z1[n - 4]);
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[k][n][r], st.unit[k], base[k]));
          if (SLIDING) x[k][n][r] = p;
          l[k] += p;
          float yy = __builtin_fmaf(p, (float)sz[0], 0.0f);
          const bool coded = !SLIDING || 16 * n + t < fp16_from;
          y[u] = coded ? yy : 0.0f;
          zs[k] = coded ? __builtin_fmaf(p, (float)sz[1], zs[k]) : zs[k];
        }
        const half2_t w = pack_h2(y[0], y[1]);
        ys[k] = __builtin_amdgcn_fdot2(w, ones, ys[k], false);
        P[k][s][2 * r] = w[0];
        P[k][s][2 * r + 1] = w[1];
      }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    st.l[k] += l[k];
    st.mid[k] += fmaf(ys[k] * scale, Rec<BITS>::kCentre, zs[k]);
  }
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      uint32_t e0[BITS / 2], o0[BITS / 2], e1[BITS / 2], o1[BITS / 2];
#pragma unroll
      for (int pl = 0; pl < BITS / 2; ++pl) {
        const Nibbles a = nibbles_of(rec.vw[4 * pl + m][2 * hf]), b = nibbles_of(rec.vw[4 * pl + m][2 * hf + 1]);
        e0[pl] = a.first; o0[pl] = a.second; e1[pl] = b.first; o1[pl] = b.second;
      }
      half8_t V[4];
      V[0] = as_h8(code_pair<BITS, 0>(e0, scale), code_pair<BITS, 0>(o0, scale), code_pair<BITS, 0>(e1, scale), code_pair<BITS, 0>(o1, scale));
      V[1] = as_h8(code_pair<BITS, 1>(e0, scale), code_pair<BITS, 1>(o0, scale), code_pair<BITS, 1>(e1, scale), code_pair<BITS, 1>(o1, scale));
      V[2] = as_h8(code_pair<BITS, 2>(e0, scale), code_pair<BITS, 2>(o0, scale), code_pair<BITS, 2>(e1, scale), code_pair<BITS, 2>(o1, scale));
      V[3] = as_h8(code_pair<BITS, 3>(e0, scale), code_pair<BITS, 3>(o0, scale), code_pair<BITS, 3>(e1, scale), code_pair<BITS, 3>(o1, scale));
#pragma unroll
      for (int k = 0; k < NR; ++k)
#pragma unroll
        for (int s = 0; s < 4; ++s) st.acc[k][2 * m + hf] = __builtin_amdgcn_mfma_f32_16x16x32_f16(V[s], P[k][s], st.acc[k][2 * m + hf], 0, 0, 0);
    }
  if (SLIDING && fp16_from < kGroup) {
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * n + token_order(4 * (lane >> 4) + r) < fp16_from) x[k][n][r] = 0.0f;
    window_values<NR, 8>(st, v_win, quads, 0, x, lane);
  }
}

// Scores of up to 32 raw key rows of 128 halves, `count` of them there; x[k][0..1].  Rows beyond count take the last one's keys.
template <int NR>
__device__ __forceinline__ void raw_scores(Rows<NR>& st, const half_t* keys, int at, int count, int sinks, int lane, float (&x)[NR][2][4]) {
  const int g = lane >> 4;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const uint4* row = reinterpret_cast<const uint4*>(keys + (long long)min(16 * n + token_order(lane & 15), count - 1) * kHeadDim + 32 * g);
    half8_t K[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) K[s] = as_h8(row[s]);
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(K[s], st.q[k][s], d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[k][n][r] = seen(16 * n + token_order(4 * g + r), at, count, st.p[k], st.low[k], sinks) ? d[r] * st.unit[k] : -INFINITY;
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    float mx = x[k][0][0];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[k][n][r]);
    set_reference<NR>(st, k, mx);
    const float m = finite_reference(st.m[k]);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[k][n][r] = __builtin_amdgcn_exp2f(x[k][n][r] - m);
        st.l[k] += x[k][n][r];
      }
  }
}

// O^T += V^T P^T with raw value rows of 128 halves.  A lane gathers the 8 values of a channel (16 lanes: 32 contiguous bytes a row).
template <int NR>
__device__ __forceinline__ void raw_values(Rows<NR>& st, const half_t* values, int count, const float (&w)[NR][2][4], int lane) {
  const int g = lane >> 4;
  half8_t P[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k)
    P[k] = as_h8(pack_h2(w[k][0][0], w[k][0][1]), pack_h2(w[k][0][2], w[k][0][3]), pack_h2(w[k][1][0], w[k][1][1]), pack_h2(w[k][1][2], w[k][1][3]));
  const half_t* row[8];
#pragma unroll
  for (int u = 0; u < 8; ++u)
    row[u] = values + (long long)min(16 * (u >> 2) + token_order(4 * g + (u & 3)), count - 1) * kHeadDim + (lane & 15);
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    half8_t V;
#pragma unroll
    for (int u = 0; u < 8; ++u) V[u] = row[u][16 * n];
#pragma unroll
    for (int k = 0; k < NR; ++k) st.acc[k][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(V, P[k], st.acc[k][n], 0, 0, 0);
  }
}

// acc H: channels 16 n + 4 g + r, seven butterfly stages and the factor 1 / sqrt(128), in binary32.
template <int NR>
__device__ __forceinline__ void rotate_rows(Rows<NR>& st, int lane) {
  const float s16 = (lane & 16) != 0 ? -1.0f : 1.0f, s32 = (lane & 32) != 0 ? -1.0f : 1.0f;
#pragma unroll
  for (int k = 0; k < NR; ++k) {
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float4_t v = st.acc[k][n];
      const float a0 = v[0] + v[1], a1 = v[0] - v[1], a2 = v[2] + v[3], a3 = v[2] - v[3];
      float t[4] = {a0 + a2, a1 + a3, a0 - a2, a1 - a3};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x, y;
        pair_across<16>(t[r], x, y);
        t[r] = __builtin_fmaf(y, s16, x);
        pair_across<32>(t[r], x, y);
        st.acc[k][n][r] = __builtin_fmaf(y, s32, x) * kInvSqrtD;
      }
    }
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
#pragma unroll
      for (int n = 0; n < 8; ++n)
        if ((n & h) == 0) {
          const float4_t a = st.acc[k][n], b = st.acc[k][n + h];
          st.acc[k][n] = a + b;
          st.acc[k][n + h] = a - b;
        }
  }
}

// One output row from its 128 numerators (16 lanes, 8 neighbouring channels each) and the correction, if any: normalised, rotated back.
__device__ __forceinline__ void finish_row(float (&a)[8], float l, float m, const float* corr, int lane, half_t* out) {
  if (corr != nullptr) {  // {C_d, -, -, -, C_n[128]}: added as e^0 terms (Eq. 5), both sides relative to max(m, 0)
    const float to = fmaxf(m, 0.0f);
    const float f = __builtin_amdgcn_exp2f(m - to), w = __builtin_amdgcn_exp2f(-to);
    l = fmaf(w, corr[0], l * f);
    const float4 c0 = *reinterpret_cast<const float4*>(corr + 4 + 8 * (lane & 15)), c1 = *reinterpret_cast<const float4*>(corr + 8 + 8 * (lane & 15));
    const float c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = fmaf(w, c[i], a[i] * f);
  }
  lane8_butterflies(a);
  row16_butterflies<8>(a, lane);
  const float inv = l > 0.0f ? kInvSqrtD / l : 0.0f;
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = as_u32(pack_h2(a[2 * i] * inv, a[2 * i + 1] * inv));
  *reinterpret_cast<uint4*>(out + 8 * (lane & 15)) = make_uint4(h[0], h[1], h[2], h[3]);
}

struct RowPlace {
  int i, h;  // token of the call, head of the KV head
};
__device__ __forceinline__ RowPlace row_place(int row, int gq) {
  const int i = row / gq;
  return RowPlace{i, row - i * gq};
}

// Grid, one-dimensional: split fastest, then (sequence, KV head), then the block of 16 NR rows.  PROMPT: rows are new tokens at positions total + i, and see their own rows; else one
// token at position total - 1.
template <int BITS, int NR, bool PROMPT, bool SLIDING>
__global__ __launch_bounds__(64 * kRowWaves, 2) void rows_kernel(ContextCall a) {
  __shared__ __align__(16) u32x4_t sMeta[kRowWaves][64];
  const kvlinc_cache& c = a.cache;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int pairs = c.B * c.H_kv, unit = blockIdx.x / a.splits, split = blockIdx.x - unit * a.splits;
  const int block = unit / pairs, bh = unit - block * pairs, b = bh / c.H_kv, kvh = bh - b * c.H_kv, gq = a.gq;
  const Lengths len = lengths_of(c, b);
  const int T = PROMPT ? (a.n_new != nullptr ? min(max(a.n_new[b], 0), a.T) : a.T) : 1;
  const int rows = T * gq, row0 = block * 16 * NR;
  if (row0 >= rows) return;
  const int total = len.total(), base = PROMPT ? total : total - 1;
  const long long head0 = (long long)b * c.H_q + (long long)kvh * gq;

  Rows<NR> st;
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const RowPlace at = row_place(min(row0 + 16 * k + (lane & 15), rows - 1), gq);
    st.p[k] = base + at.i;
    st.low[k] = window_low(st.p[k], a.window);
    const uint4* src = reinterpret_cast<const uint4*>(a.q + ((head0 + at.h) * a.T + at.i) * kHeadDim + 32 * g);
    uint4 raw[4];
    uint32_t mx = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      raw[s] = src[s];
      const uint32_t w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = max(mx, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    }
    const auto u = __builtin_amdgcn_permlane16_swap(mx, mx, false, false);
    mx = max(u[0], u[1]);
    const auto v = __builtin_amdgcn_permlane32_swap(mx, mx, false, false);
    mx = max(v[0], v[1]);
    const int e = (int)min(max(mx >> 10, 1u), 30u) - 14;  // largest magnitude in [2^(e-1), 2^e) (subnormal rows: below 2^-14, e = -13)
    const float down = bits_f32((uint32_t)(127 - e) << 23);
    st.unit[k] = bits_f32((uint32_t)(127 + e) << 23) * kLog2eSqrtD;
    const half2_t down2 = pack_h2(down, down);
#pragma unroll
    for (int s = 0; s < 4; ++s)
      st.q[k][s] = as_h8(as_h2(raw[s].x) * down2, as_h2(raw[s].y) * down2, as_h2(raw[s].z) * down2, as_h2(raw[s].w) * down2);
    st.m[k] = -INFINITY;
    st.l[k] = st.mid[k] = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) st.acc[k][n] = float4_t{0.f, 0.f, 0.f, 0.f};
  }

  // Blocks of tokens that some row sees: the new rows' (32 each), the window's (32 each), the groups.  `low` is that of the first row, the
  // last row's position ends the new ones.
  const int first_i = row0 / gq, last_i = min(row0 + 16 * NR - 1, rows - 1) / gq;
  const int low = window_low(base + first_i, a.window), low_last = window_low(base + last_i, a.window);
  const int new_from = PROMPT ? (a.sinks > total ? 0 : max(low - total, 0) / kRawTokens) : 0;
  const int n_new = PROMPT ? (last_i + kRawTokens) / kRawTokens - new_from : 0;
  const int win_from = a.sinks > len.nq ? 0 : min(max(low - len.nq, 0), len.nr) / kRawTokens;
  const int n_win = (len.nr + kRawTokens - 1) / kRawTokens - win_from;
  const int G = len.groups(), group_low = min(low / kGroup, G);
  const int n_sink = a.window > 0 ? min((int)(((long long)a.sinks + kGroup - 1) / kGroup), group_low) : 0;
  const int n_groups = G - group_low + n_sink;
  const int step = kRowWaves * a.splits;
  int item = split * kRowWaves + wave;

  if (PROMPT) {
    bool rotate = false;
    const half_t* keys = a.k_new + (long long)bh * a.T * kHeadDim;
    const half_t* values = a.v_new + (long long)bh * a.T * kHeadDim;
    for (; item < n_new; item += step) {
      const int t0 = (new_from + item) * kRawTokens;
      float x[NR][2][4];
      raw_scores<NR>(st, keys + (long long)t0 * kHeadDim, total + t0, min(T - t0, kRawTokens), a.sinks, lane, x);
      raw_values<NR>(st, values + (long long)t0 * kHeadDim, min(T - t0, kRawTokens), x, lane);
      rotate = true;
    }
    if (rotate) rotate_rows<NR>(st, lane);  // from here on the accumulators are in the cache's rotated basis
  }
  item -= n_new;
  const half_t* k_win = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
  const half_t* v_win = reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim;
  const int quads = c.R / 4;
  for (; item < n_win; item += step) {
    const int t0 = (win_from + item) * kRawTokens;
    float x[NR][2][4];
    raw_scores<NR>(st, k_win + t0 * kHeadDim, len.nq + t0, min(len.nr - t0, kRawTokens), a.sinks, lane, x);
    window_values<NR, 2>(st, v_win, quads, t0 / 16, x, lane);
  }
  item -= n_win;
  const uint32_t* rec0 = c.groups + (long long)bh * c.max_groups * Rec<BITS>::kWords;
  const int newest = SLIDING && len.nq % kGroup == 0 && len.nr < kGroup ? G - 1 : -1;
  auto group_of = [&](int it) { return it < n_sink ? it : it - n_sink + group_low; };
  if (item < n_groups) {
    Record<BITS> rec;
    int gr = group_of(item);
    load_key_part<BITS>(rec, rec0 + (long long)gr * Rec<BITS>::kWords, lane);
    load_value_part<BITS>(rec, rec0 + (long long)gr * Rec<BITS>::kWords, lane);
    for (;;) {
      const int at = gr * kGroup, count = min(len.nq - at, kGroup);
      const bool masked = count < kGroup || (at < low_last && at + kGroup > a.sinks), more = item + step < n_groups;
      const int e = put_meta<BITS>(rec, sMeta[wave], lane);
      float x[NR][8][4], exponent_base[NR];
      group_scores<BITS, NR>(st, rec, sMeta[wave], at, count, masked, a.sinks, lane, x, exponent_base);
      const int next = more ? group_of(item + step) : gr;
      if (more) load_key_part<BITS>(rec, rec0 + (long long)next * Rec<BITS>::kWords, lane);
      group_values<BITS, NR, SLIDING>(st, rec, sMeta[wave], e, x, exponent_base, gr == newest ? len.nr : kGroup, v_win, quads, lane);
      if (!more) break;
      load_value_part<BITS>(rec, rec0 + (long long)next * Rec<BITS>::kWords, lane);
      item += step;
      gr = next;
    }
  }

  // ---- the four waves joined ----
  constexpr int kAccStride = kHeadDim + 4;
  __shared__ float sM[kRowWaves][16 * NR], sL[kRowWaves][16 * NR];
  __shared__ __align__(16) float sAcc[kRowWaves][16][kAccStride];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    float l = st.l[k], mid = st.mid[k], x, y;
    pair_across<16>(l, x, y);
    pair_across<32>(x + y, x, y);
    l = x + y;
    pair_across<16>(mid, x, y);
    pair_across<32>(x + y, x, y);
    mid = x + y;
    if (g == 0) { sM[wave][16 * k + lane] = st.m[k]; sL[wave][16 * k + lane] = l; }
    if (k > 0) __syncthreads();
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float4_t v = st.acc[k][n];
      *reinterpret_cast<float4*>(&sAcc[wave][lane & 15][16 * n + 4 * g]) = make_float4(v[0] + mid, v[1] + mid, v[2] + mid, v[3] + mid);
    }
    __syncthreads();
    const int r = 16 * k + (threadIdx.x >> 4), row = row0 + r, ch = 8 * (lane & 15);
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) M = fmaxf(M, sM[w][r]);
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, L = 0.0f;
    if (M != -INFINITY) {
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sM[w][r] - M);  // 0 for a wave that has seen nothing
        L = fmaf(f, sL[w][r], L);
        const float4 u0 = *reinterpret_cast<const float4*>(&sAcc[w][r - 16 * k][ch]), u1 = *reinterpret_cast<const float4*>(&sAcc[w][r - 16 * k][ch + 4]);
        o[0] = fmaf(f, u0.x, o[0]); o[1] = fmaf(f, u0.y, o[1]); o[2] = fmaf(f, u0.z, o[2]); o[3] = fmaf(f, u0.w, o[3]);
        o[4] = fmaf(f, u1.x, o[4]); o[5] = fmaf(f, u1.y, o[5]); o[6] = fmaf(f, u1.z, o[6]); o[7] = fmaf(f, u1.w, o[7]);
      }
    }
    if (row < rows) {
      const RowPlace at = row_place(row, gq);
      const long long place = (head0 + at.h) * a.T + at.i;
      if (a.splits == 1) {
        finish_row(o, L, M, a.corr != nullptr ? a.corr + place * kPartStride : nullptr, lane, a.out + place * kHeadDim);
      } else {
        float* dst = a.part + (place * a.splits + split) * kPartStride;
        if ((lane & 15) == 0) { dst[0] = M; dst[1] = L; }
        *reinterpret_cast<float4*>(dst + 4 + ch) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(dst + 8 + ch) = make_float4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

// The splits of 16 rows joined, 16 lanes a row.  Row = ((b H_kv + g) gq + h) T + i.
template <bool PROMPT>
__global__ __launch_bounds__(256) void join_kernel(ContextCall a, long long n_rows) {
  const int lane = threadIdx.x & 63;
  const long long place = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (place >= n_rows) return;
  if (PROMPT && a.n_new != nullptr) {
    const long long h = place / a.T;
    if (place - h * a.T >= a.n_new[h / a.cache.H_q]) return;
  }
  const float* p = a.part + place * a.splits * kPartStride;
  float M = -INFINITY;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, p[s * kPartStride]);
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, L = 0.0f;
  if (M != -INFINITY)
    for (int s = 0; s < a.splits; ++s) {
      const float* src = p + s * kPartStride;
      const float f = __builtin_amdgcn_exp2f(src[0] - M);
      L = fmaf(f, src[1], L);
      const float4 u0 = *reinterpret_cast<const float4*>(src + 4 + 8 * (lane & 15)), u1 = *reinterpret_cast<const float4*>(src + 8 + 8 * (lane & 15));
      o[0] = fmaf(f, u0.x, o[0]); o[1] = fmaf(f, u0.y, o[1]); o[2] = fmaf(f, u0.z, o[2]); o[3] = fmaf(f, u0.w, o[3]);
      o[4] = fmaf(f, u1.x, o[4]); o[5] = fmaf(f, u1.y, o[5]); o[6] = fmaf(f, u1.z, o[6]); o[7] = fmaf(f, u1.w, o[7]);
    }
  finish_row(o, L, M, a.corr != nullptr ? a.corr + place * kPartStride : nullptr, lane, a.out + place * kHeadDim);
}

}  // namespace

template <int BITS, int NR, bool PROMPT>
static void launch_rows_of(const ContextCall& a, dim3 grid, hipStream_t stream) {
  const bool sliding = (a.cache.flags & KVLINC_FLAG_SLIDING_VALUES) != 0;
  if (sliding) hipLaunchKernelGGL((rows_kernel<BITS, NR, PROMPT, true>), grid, dim3(64 * kRowWaves), 0, stream, a);
  else hipLaunchKernelGGL((rows_kernel<BITS, NR, PROMPT, false>), grid, dim3(64 * kRowWaves), 0, stream, a);
}

int launch_rows(const ContextCall& a, bool prompt, hipStream_t stream) {
  const long long rows = (long long)a.T * a.gq;
  const dim3 grid((unsigned)(a.splits * (long long)a.cache.B * a.cache.H_kv * ((rows + 15) / 16)));
  if (a.cache.bits == 2) prompt ? launch_rows_of<2, 1, true>(a, grid, stream) : launch_rows_of<2, 1, false>(a, grid, stream);
  else prompt ? launch_rows_of<4, 1, true>(a, grid, stream) : launch_rows_of<4, 1, false>(a, grid, stream);
  if (hipGetLastError() != hipSuccess) return KVLINC_EHIP;
  return a.splits > 1 ? launch_join(a, prompt, stream) : KVLINC_OK;
}

int launch_join(const ContextCall& a, bool prompt, hipStream_t stream) {
  const long long n = (long long)a.cache.B * a.cache.H_q * a.T;
  const dim3 grid((unsigned)((n + 15) / 16));
  if (prompt) hipLaunchKernelGGL(join_kernel<true>, grid, dim3(256), 0, stream, a, n);
  else hipLaunchKernelGGL(join_kernel<false>, grid, dim3(256), 0, stream, a, n);
  return hipGetLastError() == hipSuccess ? KVLINC_OK : KVLINC_EHIP;
}

}  // namespace kvlinc
