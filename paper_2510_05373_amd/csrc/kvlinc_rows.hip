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
#include "kvlinc_reference.h"

namespace kvlinc {
namespace {

constexpr int kMaxWaves = 8;
constexpr int kRawTokens = 32;
// Columns of the products: 16 rows of queries; or, of up to 8 or 4 rows, each row S = 2 or 4 times, column c with row c % (16 / S) and subset
// c / (16 / S): the softmax of a column is then over the 16-token blocks n with n / (8 / S) = subset only, and a lane has 8 / S blocks' scores to
// work on instead of 8.
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
// value (scale, middle) of tokens 16 (4 u + i) + t, i = 0..3, the middle z + centre s in binary16: a value is s (code - centre) + middle, and a
// weight's rounding counts with the first part only.  Returned: the exponent e of the group's largest value scale, which goes from the weights to the
// codes (2^-e weight scale stays in binary16's range whatever the values' magnitude, and the codes times 2^e are exact), and the bits of the largest key scale.
struct GroupMagnitudes {
  int value_exponent;
  uint32_t key_scale;
};
template <int BITS>
__device__ __forceinline__ GroupMagnitudes put_meta(const Record<BITS>& r, u32x4_t* meta, int lane) {
  // scales are not negative: their bit patterns order like the numbers
  typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
  const auto halves = [&](int i) {
    const uint32_t w = r.meta[i];  // (a bit cast of r.meta[i] itself would take r.meta[0]: it goes by the address of the vector)
    return __builtin_bit_cast(ushort2_t, w);
  };
  const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_max(halves(0), halves(1)), __builtin_elementwise_max(halves(2), halves(3))));
  uint32_t top = lane >= 32 ? both & 0xffffu : max(both & 0xffffu, both >> 16);  // (lanes 0..15: key scales; 32..63: value scales)
  top = max(top, dpp_u<kRowRor1>(top));
  top = max(top, dpp_u<kRowRor2>(top));
  top = max(top, dpp_u<kRowRor4>(top));
  top = max(top, dpp_u<kRowRor8>(top));
  const int e = (int)(max(max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)) >> 10, 3u)) - 15;  // -12 .. 15: the codes times 2^e are normal numbers
  const half_t centre = (half_t)(lane >= 32 ? Rec<BITS>::kCentre : 0.0f);
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half2_t v = as_h2(r.meta[i]);
    w[i] = as_u32(half2_t{v[0], __builtin_elementwise_fma(v[0], centre, v[1])});
  }
  meta[lane] = w;
  __builtin_amdgcn_wave_barrier();  // (a wave's LDS instructions stay in order)
  return GroupMagnitudes{e, (uint32_t)__builtin_amdgcn_readlane(top, 0)};
}

// Queries are scaled to have their largest magnitude in [2^5, 2^6): as small as binary16 can hold beside it are then 2^-30 of it, and products with key
// scales below 2^10 stay below 65504.
constexpr int kQueryTop = 6;
constexpr uint32_t kFirstLargeScale = (15 + 16 - kQueryTop) << 10;  // 2^10 in binary16
struct Rows {
  half8_t q[4];       // query of this lane's row, channels 32 g + 8 step .. + 7, scaled
  float unit;      // log2(e) / sqrt(d) over that scale
  bool lossy;      // some query of the wave's rows is not held exactly (the same in all lanes)
  int p, low;      // position, first token of its window
  int subset;
  float m;         // reference (the same in the four lanes of a column), log2 domain; -inf: nothing seen yet
  float l, mid;    // per-lane sums of the weights, and of weight times middle: the same for all channels
  float4_t acc[8]; // numerator of channels 16 n + 4 g + 0..3
};

// Token of register r, block n of the tile whose first token is `at`, or -1 beyond its `count` tokens; and whether a row sees it.
__device__ __forceinline__ bool seen(int t, int at, int count, int p, int low, int sinks) {
  const int pos = at + t;
  return t < count && pos <= p && (pos >= low || pos < sinks);
}

__device__ __forceinline__ void set_reference(Rows& st, float largest) {  // largest: of this lane's scores
  if (__builtin_amdgcn_ballot_w64(passes(largest, st.m)) == 0) return;
  float x, y;
  pair_across<16>(largest, x, y);
  pair_across<32>(fmaxf(x, y), x, y);
  const float to = raised(fmaxf(x, y), st.m), f = raised_factor(st.m, to);
  st.m = to;
  st.l *= f;
  st.mid *= f;
#pragma unroll
  for (int n = 0; n < 8; ++n) st.acc[n] *= f;
}
__device__ __forceinline__ float finite_reference(float m) { return m == -INFINITY ? 0.0f : m; }

// O^T += V^T P^T with the window's fp16 values of the 16-token blocks first .. first + NB - 1 (two a product), weights w[n][r] by block.
// v_res is [slot / 4][channel][slot % 4]: a lane takes two neighbouring slots at a time.
template <int NB>
__device__ __forceinline__ void window_values(Rows& st, const half_t* v_win, int quads, int first, const float (&w)[NB][4], int lane) {
  const int g = lane >> 4, a = 8 * (g & 1) + 2 * (g >> 1);
#pragma unroll
  for (int s = 0; s < NB / 2; ++s) {
    const half8_t P = as_h8(pack_h2(w[2 * s][0], w[2 * s][1]), pack_h2(w[2 * s][2], w[2 * s][3]), pack_h2(w[2 * s + 1][0], w[2 * s + 1][1]),
                            pack_h2(w[2 * s + 1][2], w[2 * s + 1][3]));
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      u32x4_t v;
#pragma unroll
      for (int u = 0; u < 4; ++u) {  // (slots beyond the window take its last quad's: their weights are 0 and the window is finite)
        const int slot = 16 * (first + 2 * s + (u >> 1)) + a + 4 * (u & 1);
        v[u] = *reinterpret_cast<const uint32_t*>(v_win + ((long long)min(slot >> 2, quads - 1) * kHeadDim + 16 * n + (lane & 15)) * 4 + (slot & 3));
      }
      st.acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(v), P, st.acc[n], 0, 0, 0);
    }
    asm volatile("" ::: "memory");  // (the next blocks' loads stay behind these products: all at once they spilled)
  }
}

// The operands of a group's first product from the query as it is (q_row: this lane's channels): products with the key scales in binary32, the largest of
// a row brought to [2^14, 2^15).  For queries whose smallest binary16 would lose beside the largest (one of 64 or more is needed for
// that), and key scales from 2^10 on.  A call takes 10 to 16 % longer so (16 sequences of 8k tokens, 4 rows: 27.5 and 31.3 us; 6 over 131072: 50 and 58).
template <int BITS>
__device__ __forceinline__ void wide_operands(const half_t* q_row, const u32x4_t* meta, int lane, half8_t (&hi)[4], half8_t (&lo)[4], float& bias, float& unit) {
  u32x4_t q[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) q[s] = reinterpret_cast<const u32x4_t*>(q_row)[s];
  float mx = 0.0f, bz = 0.0f, bs = 0.0f;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const u32x4_t sc = meta[4 * (lane >> 4) + s], z = meta[16 + 4 * (lane >> 4) + s];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const half2_t a = as_h2(q[s][i]), k = as_h2(sc[i]);
      mx = fmaxf(mx, fmaxf(fabsf((float)a[0] * (float)k[0]), fabsf((float)a[1] * (float)k[1])));
      bz = __builtin_amdgcn_fdot2(a, as_h2(z[i]), bz, false);
      bs = __builtin_amdgcn_fdot2(a, k, bs, false);
    }
  }
  float a, b;
  pair_across<16>(fmaf(bs, Rec<BITS>::kCentre, bz), a, b);
  pair_across<32>(a + b, a, b);
  bias = (a + b) * kLog2eSqrtD;
  pair_across<16>(mx, a, b);
  pair_across<32>(fmaxf(a, b), a, b);
  const uint32_t e = max(__builtin_bit_cast(uint32_t, fmaxf(a, b)) >> 23, 87u);  // (2^-40 at least: none is below 2^-48, and it may be 0)
  const float scale = bits_f32((254u + 14u - e) << 23);
  unit = bits_f32((e - 14u) << 23) * kLog2eSqrtD;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const u32x4_t sc = meta[4 * (lane >> 4) + s];
    u32x4_t h, r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const half2_t a = as_h2(q[s][i]), k = as_h2(sc[i]);
      const float p0 = (float)a[0] * (float)k[0] * scale, p1 = (float)a[1] * (float)k[1] * scale;
      const half2_t t = pack_h2(p0, p1);
      h[i] = as_u32(t);
      r[i] = as_u32(pack_h2(p0 - (float)t[0], p1 - (float)t[1]));
    }
    hi[s] = as_h8(h);
    lo[s] = as_h8(r);
  }
}

// Scores of one group of 128 packed tokens, the first at position `at`, `count` of them there: x[i][r] = block subset (8 / S) + i, token
// 16 n + pi(4 g + r), and with `base` the exponent of a weight, x unit + base.  masked: some row does not see all of them.
template <int BITS, int S, typename Q>
__device__ __forceinline__ void group_scores(Rows& st, const Record<BITS>& rec, const u32x4_t* meta, uint32_t key_scale, Q q_row, int at, int count, bool masked, int sinks, int lane,
                                             float (&x)[8 / S][4], float& unit, float& base) {
  constexpr int kBlocks = 8 / S;
  half8_t hi[4], lo[4];
  float bias;
  if (st.lossy || key_scale >= kFirstLargeScale) {
    wide_operands<BITS>(q_row(), meta, lane, hi, lo, bias, unit);
  } else {
    unit = st.unit;
    float bz = 0.0f, bs = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4_t sc = meta[4 * (lane >> 4) + s], z = meta[16 + 4 * (lane >> 4) + s];
      const u32x4_t qq = __builtin_bit_cast(u32x4_t, st.q[s]);
      u32x4_t h, r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const half2_t a = as_h2(qq[i]), k = as_h2(sc[i]), t = a * k;
        h[i] = as_u32(t);
        r[i] = as_u32(__builtin_elementwise_fma(a, k, -t));
        bz = __builtin_amdgcn_fdot2(a, as_h2(z[i]), bz, false);
        bs = __builtin_amdgcn_fdot2(a, k, bs, false);
      }
      hi[s] = as_h8(h);
      lo[s] = as_h8(r);
    }
    float a, b;
    pair_across<16>(fmaf(bs, Rec<BITS>::kCentre, bz), a, b);
    pair_across<32>(a + b, a, b);
    bias = (a + b) * st.unit;
  }
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    half8_t A[4];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
      for (int pl = 0; pl < BITS / 2; ++pl) {
        const Nibbles nb = nibbles_of(rec.kw[4 * pl + n / 2][2 * (n % 2) + w]);
        e[pl] = nb.first; o[pl] = nb.second;
      }
      A[2 * w] = as_h8(code_pair<BITS, 0>(e, 1.0f), code_pair<BITS, 1>(e, 1.0f), code_pair<BITS, 2>(e, 1.0f), code_pair<BITS, 3>(e, 1.0f));
      A[2 * w + 1] = as_h8(code_pair<BITS, 0>(o, 1.0f), code_pair<BITS, 1>(o, 1.0f), code_pair<BITS, 2>(o, 1.0f), code_pair<BITS, 3>(o, 1.0f));
    }
    float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[s], lo[s], d, 0, 0, 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(A[s], hi[s], d, 0, 0, 0);
    const bool own = S == 1 || n / kBlocks == st.subset;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[n % kBlocks][r] = n < kBlocks || own ? d[r] : x[n % kBlocks][r];
  }
  if (masked) {
    const int t0 = 16 * kBlocks * st.subset, end = min(count, st.p - at + 1) - t0, from = st.low - at - t0, first = sinks - at - t0;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + token_order(4 * (lane >> 4) + r);
        x[i][r] = (t < end) & ((t >= from) | (t < first)) ? x[i][r] : -INFINITY;
      }
  }
  float mx = x[0][0];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[i][r]);
  set_reference(st, fmaf(mx, unit, bias));
  const float m = finite_reference(st.m);
  base = bias - m;
  // References and biases thousands beyond what ordinary keys and queries give: the exponents are rounded as the reference was (the score
  // itself, then its distance from the reference), or the exponent of the largest weight would be what the roundings leave.
  if (__builtin_amdgcn_ballot_w64(fmaxf(fabsf(m), fabsf(bias)) > kFusedBound) != 0) {
#pragma clang fp contract(off)
    const float back = 1.0f / unit;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[i][r] = (__builtin_fmaf(x[i][r], unit, bias) - m) * back;
    base = 0.0f;
  }
}

// Scores become weights; O^T += V^T P^T of the group.  e: value_exponent of put_meta.  SLIDING: tokens from fp16_from on take their values from the window.
template <int BITS, int S, bool SLIDING>
__device__ __forceinline__ void group_values(Rows& st, const Record<BITS>& rec, const u32x4_t* meta, int e, float (&x)[8 / S][4], float unit, float base, int fp16_from,
                                             const half_t* v_win, int quads, int lane) {
  constexpr int kBlocks = 8 / S;
  const float scale = bits_f32((uint32_t)(127 + e) << 23);
  base -= (float)e;  // weights here: times 2^-e
  uint32_t w[kBlocks / 2][4];  // weight times value scale of blocks 2 i and 2 i + 1
  float l = 0.0f, mid = 0.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = token_order(4 * (lane >> 4) + r);
    const uint32_t* pairs = reinterpret_cast<const uint32_t*>(meta + 32 + 2 * t) + kBlocks * st.subset;
    uint32_t sz[kBlocks];
    if constexpr (S == 4) {
      const u32x2_t v = *reinterpret_cast<const u32x2_t*>(pairs);
      sz[0] = v[0]; sz[1] = v[1];
    } else {
#pragma unroll
      for (int q = 0; q < kBlocks / 4; ++q) {
        const u32x4_t v = reinterpret_cast<const u32x4_t*>(pairs)[q];
#pragma unroll
        for (int i = 0; i < 4; ++i) sz[4 * q + i] = v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kBlocks; i += 2) {
      float y[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const half2_t p2 = as_h2(sz[i + u]);
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i + u][r], unit, base));
        if (SLIDING) x[i + u][r] = p * scale;
        l += p;
        const bool coded = !SLIDING || 16 * (kBlocks * st.subset + i + u) + t < fp16_from;
        const float yy = __builtin_fmaf(p, (float)p2[0], 0.0f);
        y[u] = coded ? yy : 0.0f;
        mid = coded ? __builtin_fmaf(p, (float)p2[1], mid) : mid;
      }
      w[i / 2][r] = as_u32(pack_h2(y[0], y[1]));
    }
  }
  st.l = fmaf(l, scale, st.l);
  st.mid = fmaf(mid, scale, st.mid);
  half8_t P[4];  // step s: blocks 2 s and 2 s + 1; a column has those of its subset, and zero elsewhere
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    u32x4_t v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = S == 1 || 2 * s / kBlocks == st.subset ? w[s % (kBlocks / 2)][r] : 0u;
    P[s] = as_h8(v);
  }
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    uint32_t e0[BITS / 2], o0[BITS / 2], e1[BITS / 2], o1[BITS / 2];
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles a = nibbles_of(rec.vw[4 * pl + n / 2][2 * (n % 2)]), b = nibbles_of(rec.vw[4 * pl + n / 2][2 * (n % 2) + 1]);
      e0[pl] = a.first; o0[pl] = a.second; e1[pl] = b.first; o1[pl] = b.second;
    }
    half8_t V[4];
    V[0] = as_h8(code_pair<BITS, 0>(e0, scale), code_pair<BITS, 0>(o0, scale), code_pair<BITS, 0>(e1, scale), code_pair<BITS, 0>(o1, scale));
    V[1] = as_h8(code_pair<BITS, 1>(e0, scale), code_pair<BITS, 1>(o0, scale), code_pair<BITS, 1>(e1, scale), code_pair<BITS, 1>(o1, scale));
    V[2] = as_h8(code_pair<BITS, 2>(e0, scale), code_pair<BITS, 2>(o0, scale), code_pair<BITS, 2>(e1, scale), code_pair<BITS, 2>(o1, scale));
    V[3] = as_h8(code_pair<BITS, 3>(e0, scale), code_pair<BITS, 3>(o0, scale), code_pair<BITS, 3>(e1, scale), code_pair<BITS, 3>(o1, scale));
#pragma unroll
    for (int s = 0; s < 4; ++s) st.acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(V[s], P[s], st.acc[n], 0, 0, 0);
  }
  if (SLIDING && fp16_from < kGroup) {
    float p[8][4];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        p[n][r] = (S == 1 || n / kBlocks == st.subset) && 16 * n + token_order(4 * (lane >> 4) + r) >= fp16_from ? x[n % kBlocks][r] : 0.0f;
    window_values<8>(st, v_win, quads, 0, p, lane);
  }
}

// Weights of up to 32 raw key rows of 128 halves, `count` of them there (all in subset 0).  Rows beyond count take the last one's keys.  Returns
// which of the lane's tokens its row sees, bit 4 n + r.
template <typename Q>
__device__ __forceinline__ uint32_t raw_weights(Rows& st, Q q_row, const half_t* keys, int at, int count, int sinks, int lane, float (&x)[2][4]) {
  const int g = lane >> 4;
  half8_t q[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) q[s] = st.q[s];
  float unit = st.unit;
  if (st.lossy) {
    const u32x4_t* src = reinterpret_cast<const u32x4_t*>(q_row());
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = as_h8(src[s]);
    unit = kLog2eSqrtD;
  }
  uint32_t seen_bits = 0;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const u32x4_t* row = reinterpret_cast<const u32x4_t*>(keys + (long long)min(16 * n + token_order(lane & 15), count - 1) * kHeadDim + 32 * g);
    float4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(row[s]), q[s], d, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool is = st.subset == 0 && seen(16 * n + token_order(4 * g + r), at, count, st.p, st.low, sinks);
      x[n][r] = is ? d[r] * unit : -INFINITY;
      seen_bits |= is ? 1u << (4 * n + r) : 0u;
    }
  }
  float mx = x[0][0];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[n][r]);
  set_reference(st, mx);
  const float m = finite_reference(st.m);
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[n][r] = __builtin_amdgcn_exp2f(x[n][r] - m);
      st.l += x[n][r];
    }
  return seen_bits;
}

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

struct RowPlace {
  int i, h;  // token of the call, head of the KV head
};
__device__ __forceinline__ RowPlace row_place(int row, int gq) {
  const int i = row / gq;
  return RowPlace{i, row - i * gq};
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
        const u32x4_t* src = reinterpret_cast<const u32x4_t*>(q_row());
        u32x4_t raw[4];
        uint32_t mx = 0;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          raw[s] = src[s];
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = max(mx, max(raw[s][i] & 0x7fffu, (raw[s][i] >> 16) & 0x7fffu));
        }
        const auto u = __builtin_amdgcn_permlane16_swap(mx, mx, false, false);
        mx = max(u[0], u[1]);
        const auto v = __builtin_amdgcn_permlane32_swap(mx, mx, false, false);
        mx = max(v[0], v[1]);
        const int e = (int)min(max(mx >> 10, 1u), 30u) - 14;  // largest magnitude in [2^(e-1), 2^e) (subnormal rows: below 2^-14, e = -13)
        const int shift = min(kQueryTop - e, 15);             // (2^15: binary16's largest power of two; what is so small is held exactly)
        const half2_t by = pack_h2(bits_f32((uint32_t)(127 + shift) << 23), bits_f32((uint32_t)(127 + shift) << 23));
        const half2_t back = pack_h2(bits_f32((uint32_t)(127 - shift) << 23), bits_f32((uint32_t)(127 - shift) << 23));
        st.unit = bits_f32((uint32_t)(127 - shift) << 23) * kLog2eSqrtD;
        uint32_t lost = 0;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          u32x4_t scaled;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            scaled[i] = as_u32(as_h2(raw[s][i]) * by);
            lost |= as_u32(as_h2(scaled[i]) * back) ^ raw[s][i];
          }
          st.q[s] = as_h8(scaled);
        }
        st.lossy = __builtin_amdgcn_ballot_w64(lost != 0) != 0;
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
