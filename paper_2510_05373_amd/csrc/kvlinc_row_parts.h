// A block of 16 query rows over the packed cache, a wave's work on one group of tokens at a time: what the kernels share that take few rows (not part
// of the C ABI).  The layout of the products and the arithmetic: kvlinc_rows.hip.
#pragma once

#include "kvlinc_codes.h"
#include "kvlinc_reference.h"

namespace kvlinc {
namespace {

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

// The power of two that brings a row's queries to their scale, from the bits of its largest magnitude, and the way back.
struct QueryScale {
  half2_t by, back;
  float unit;
};
__device__ __forceinline__ QueryScale query_scale(uint32_t largest) {
  const int e = (int)min(max(largest >> 10, 1u), 30u) - 14;  // largest magnitude in [2^(e-1), 2^e) (subnormal rows: below 2^-14, e = -13)
  const int shift = min(kQueryTop - e, 15);                  // (2^15: binary16's largest power of two; what is so small is held exactly)
  const float by = bits_f32((uint32_t)(127 + shift) << 23), back = bits_f32((uint32_t)(127 - shift) << 23);
  return QueryScale{pack_h2(by, by), pack_h2(back, back), back * kLog2eSqrtD};
}
// A row's query brought to its scale: q_row is what this lane takes of it.
__device__ __forceinline__ void load_query(Rows& st, const half_t* q_row, int lane) {
  const u32x4_t* src = reinterpret_cast<const u32x4_t*>(q_row);
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
  const QueryScale to = query_scale(mx);
  st.unit = to.unit;
  uint32_t lost = 0;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    u32x4_t scaled;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      scaled[i] = as_u32(as_h2(raw[s][i]) * to.by);
      lost |= as_u32(as_h2(scaled[i]) * to.back) ^ raw[s][i];
    }
    st.q[s] = as_h8(scaled);
  }
  st.lossy = __builtin_amdgcn_ballot_w64(lost != 0) != 0;
}

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

// The operands of a group's first product: query times key scales in two binary16 terms, what the zero-points and the centring add to a score (bias,
// log2 domain), and the factor of the products (unit).
template <int BITS, typename Q>
__device__ __forceinline__ void row_operands(const half8_t (&q)[4], float q_unit, bool lossy, Q q_row, const u32x4_t* meta, uint32_t key_scale, int lane, half8_t (&hi)[4],
                                             half8_t (&lo)[4], float& bias, float& unit) {
  if (lossy || key_scale >= kFirstLargeScale) {
    wide_operands<BITS>(q_row(), meta, lane, hi, lo, bias, unit);
  } else {
    unit = q_unit;
    float bz = 0.0f, bs = 0.0f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4_t sc = meta[4 * (lane >> 4) + s], z = meta[16 + 4 * (lane >> 4) + s];
      const u32x4_t qq = __builtin_bit_cast(u32x4_t, q[s]);
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
    bias = (a + b) * q_unit;
  }
}

// Keys of token block n (16 tokens) as the first product takes them, unscaled.
template <int BITS>
__device__ __forceinline__ void key_operands(const u32x4_t (&kw)[2 * BITS], int n, half8_t (&A)[4]) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    uint32_t e[BITS / 2], o[BITS / 2];
#pragma unroll
    for (int pl = 0; pl < BITS / 2; ++pl) {
      const Nibbles nb = nibbles_of(kw[4 * pl + n / 2][2 * (n % 2) + w]);
      e[pl] = nb.first; o[pl] = nb.second;
    }
    A[2 * w] = as_h8(code_pair<BITS, 0>(e, 1.0f), code_pair<BITS, 1>(e, 1.0f), code_pair<BITS, 2>(e, 1.0f), code_pair<BITS, 3>(e, 1.0f));
    A[2 * w + 1] = as_h8(code_pair<BITS, 0>(o, 1.0f), code_pair<BITS, 1>(o, 1.0f), code_pair<BITS, 2>(o, 1.0f), code_pair<BITS, 3>(o, 1.0f));
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
  row_operands<BITS>(st.q, st.unit, st.lossy, q_row, meta, key_scale, lane, hi, lo, bias, unit);
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    half8_t A[4];
    key_operands<BITS>(rec.kw, n, A);
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

struct RowPlace {
  int i, h;  // token of the call, head of the KV head
};
__device__ __forceinline__ RowPlace row_place(int row, int gq) {
  const int i = row / gq;
  return RowPlace{i, row - i * gq};
}

}  // namespace
}  // namespace kvlinc
