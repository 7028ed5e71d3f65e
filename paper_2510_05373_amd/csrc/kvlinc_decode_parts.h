// The two contractions of a group on the packed codes, the running softmax and the fp16 window, as the kernels that decode one token share
// them (kvlinc_decode.hip, which explains the arithmetic, and kvlinc_windowed.hip).  Not part of the C ABI.
#pragma once

#include "kvlinc_internal.h"
#include "kvlinc_mfma.h"
#include "kvlinc_schedule.h"

namespace kvlinc {
namespace {

constexpr int kThreads = 64 * kWaves;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kAlpha = kLog2e * 0.08838834764831845f;  // log2(e) / sqrt(128)

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short short2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

// ---- small helpers ----------------------------------------------------------------------------------------------

// Results that one workgroup writes and another reads inside the same launch (split partials, correction parts) go
// through stores and loads that are coherent across the chip's L2 slices: a workgroup-wide cache write-back /
// invalidate (what a device-scope fence costs here) would throw away the streamed records.
__device__ __forceinline__ void st_coherent(float* p, float v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ void st_coherent2(float* p, float x, float y) {  // two neighbours, 8-byte aligned
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, float2_t{x, y}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ float2 ld_coherent2(const float* p) {  // two neighbours, 8-byte aligned
  const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  return __builtin_bit_cast(float2, v);
}
// A number that the launch only reads, through the scalar cache: it does not wait behind the vector loads requested before it.
__device__ __forceinline__ int scalar_load(const int32_t* p) {
  typedef const __attribute__((address_space(4))) int32_t* constant_ptr;
  return *reinterpret_cast<constant_ptr>(reinterpret_cast<uintptr_t>(p));
}
// Cache policy of a buffer load that is coherent in the same way: sc0 and sc1.
constexpr int kCoherentLoad = 1 | 16;
constexpr int kAllLoads = 0x0f70;  // s_waitcnt vmcnt(0)

__device__ __forceinline__ float as_f32(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// Reductions with the result in every participating lane.  row: the 16 lanes of a DPP row; quad: 4 adjacent lanes;
// xrow: the 4 lanes l, l ^ 16, l ^ 32, l ^ 48 (row swaps: odd rows of one copy against even rows of the other, then
// the upper 32 lanes of one against the lower 32 of the other).  The *_umax forms take bit patterns of non-negative
// numbers, which order like the numbers themselves (one instruction per step, no NaN handling).
__device__ __forceinline__ float row_allmax(float v) {
  v = fmaxf(v, dpp_f<kRowRor1>(v));
  v = fmaxf(v, dpp_f<kRowRor2>(v));
  v = fmaxf(v, dpp_f<kRowRor4>(v));
  return fmaxf(v, dpp_f<kRowRor8>(v));
}
__device__ __forceinline__ float row_allsum(float v) {
  v += dpp_f<kRowRor1>(v);
  v += dpp_f<kRowRor2>(v);
  v += dpp_f<kRowRor4>(v);
  return v + dpp_f<kRowRor8>(v);
}
__device__ __forceinline__ uint32_t row_umax(uint32_t v) {
  v = max(v, dpp_u<kRowRor1>(v));
  v = max(v, dpp_u<kRowRor2>(v));
  v = max(v, dpp_u<kRowRor4>(v));
  return max(v, dpp_u<kRowRor8>(v));
}
__device__ __forceinline__ uint32_t quad_umax(uint32_t v) {
  v = max(v, dpp_u<kQuadSwap1>(v));
  return max(v, dpp_u<kQuadSwap2>(v));
}
__device__ __forceinline__ float quad_allsum(float v) {
  v += dpp_f<kQuadSwap1>(v);
  return v + dpp_f<kQuadSwap2>(v);
}
__device__ __forceinline__ uint32_t xrow_umax(uint32_t v) {
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}
__device__ __forceinline__ float xrow_allsum(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(as_bits(v), as_bits(v), false, false);
  v = as_f32(a[0]) + as_f32(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
  return as_f32(b[0]) + as_f32(b[1]);
}

// The compiler may not move LDS traffic of one wave across this point (the hardware keeps a wave's LDS instructions
// in order, which is all a wave needs to hand data from lane to lane through LDS).
__device__ __forceinline__ void lds_order() { asm volatile("" ::: "memory"); }

// ---- operand layouts of v_mfma_scale_f32_16x16x128_f8f6f4 (measured on gfx950) ---------------------------------------
// D:  lane l holds column l % 16, rows 4 (l / 16) + r in its 4 registers.
// B (FP4, 4 registers): lane l holds column l % 16, positions k = 32 (l / 16) + e, nibble e = 0..31 in register order.
// A (FP8, 8 registers): lane l holds row l % 16, byte e = 0..31 in register order at position
//     k = 64 (e / 16) + 16 (l / 16) + e % 16.
// Block scales (E8M0 byte, value 2^(byte - 127)): the scale operand of lane l applies to row / column l % 16 and the
// positions 32 (l / 16) .. 32 (l / 16) + 31.
//
// Roles of a lane.  As a holder of D registers ("row role"): head hd = lane / 16 of the head block, column jd.  As a
// holder of A registers: row 4 ha + ua = (head ha, term ua), quarter ga.  The A registers are built by the lanes in
// 8-byte chunks -- chunk u of (head, quarter g) = bytes 8 u .. 8 u + 7 = positions 64 (u / 2) + 16 g + 8 (u % 2) + 0..7 --
// and handed over through LDS: the builder of (head h, quarter g, chunk u) writes its three terms at
// ex[160 h + 32 term + 2 (4 g + u)], the holder of (head h, term, quarter g) reads 8 words at ex[160 h + 32 term + 8 g].
// Term 3 of every head stays zero where there are three.  Word 128 of a head carries the block exponent where builder and holder differ.
constexpr int kExHead = 160;              // words per head in an exchange region (stride 640 B: two heads cover all banks)
constexpr int kExWords = 4 * kExHead;     // one region: 4 heads
constexpr int kExExp = 128;               // word of the block exponent

// B registers from packed words: nibble = hi|0|lo|1 = FP4 (code - 1.5).  One bit-field insert per register: the code bits of the word where `pick` has ones, the constant mantissa bit elsewhere.
// `pick` is 0xAAAAAAAA held in a scalar register (see code_bits_mask) so that the insert is a single instruction.
__device__ __forceinline__ uint32_t centred_nibbles(uint32_t w, uint32_t pick) {
  return 0x11111111u ^ (pick & (w ^ 0x11111111u));  // = (w & pick) | (0x11111111 & ~pick), in the form that selects v_bfi_b32
}
__device__ __forceinline__ uint32_t code_bits_mask() {
  uint32_t m = 0xAAAAAAAAu;
  asm volatile("" : "+s"(m));  // opaque to constant folding, so that the insert stays one instruction
  return m;
}
struct Roles {
  int lane;
  int jd, hd;      // row role
  int ua, ha, ga;  // operand role
  int c0;          // first of the 8 channels whose (q * key scale) this lane builds: chunk ua of (ha, ga)
  int wq;          // where this lane writes its chunk as a builder of q K^T operands (it builds for its own quad)
  int wp;          // ... as a builder of E V operands (it builds from the probabilities it holds in the row role)
  int rd;          // where this lane reads its operand registers
  uint32_t* ex_qk;  // this wave's exchange regions
  uint32_t* ex_pv;
  uint32_t pick;    // code_bits_mask()
};

__device__ __forceinline__ Roles make_roles(int lane, uint32_t* ex_wave) {
  Roles r;
  r.lane = lane;
  r.jd = lane & 15; r.hd = lane >> 4;
  r.ua = lane & 3; r.ha = (lane >> 2) & 3; r.ga = lane >> 4;
  r.c0 = 64 * (r.ua >> 1) + 16 * r.ga + 8 * (r.ua & 1);
  r.wq = kExHead * r.ha + 2 * (4 * r.ga + r.ua);
  r.wp = kExHead * r.hd + 2 * r.jd;
  r.rd = kExHead * r.ha + 32 * r.ua + 8 * r.ga;
  r.ex_qk = ex_wave;
  r.ex_pv = ex_wave + kExWords;
  r.pick = code_bits_mask();
  return r;
}

// x[0..7] as three FP8 terms (or more): with sc = 2^e (sc_bits its binary32 pattern, e chosen so that |x| / sc < 256),
// t_k = fp8((x - what t_0 .. t_{k-1} stand for) / (sc / 16^k)), round to nearest even.  Every residual is exact in
// binary32 (the term agrees with it in its leading bits).  t[k][v] holds values 4 v .. 4 v + 3, lowest byte first.
template <int TERMS>
__device__ __forceinline__ void split_fp8(const float (&x)[8], uint32_t sc_bits, uint32_t (&t)[TERMS][2]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
  for (int k = 0; k < TERMS; ++k) {
    const float sc = as_f32(sc_bits - ((uint32_t)(4 * k) << 23));
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      short2_t w;
      asm volatile("" : "=v"(w));  // any free register: both halves are written below (a live value would be copied first)
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, r[4 * v], r[4 * v + 1], sc, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, r[4 * v + 2], r[4 * v + 3], sc, true);
      const uint32_t bits = __builtin_bit_cast(uint32_t, w);
      t[k][v] = bits;
      if (k < TERMS - 1) {
        const float2_t f0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, sc, false);
        const float2_t f1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, sc, true);
        r[4 * v] -= f0[0]; r[4 * v + 1] -= f0[1];
        r[4 * v + 2] -= f1[0]; r[4 * v + 3] -= f1[1];
      }
    }
  }
}

// Biased binary32 exponent eb of the largest magnitude of a block, from its bit pattern (kept away from the low end of
// the range), for sc = 2^(eb - 127 - 7): |x| / sc < 256, inside FP8's range.  Row `term` then carries the block scale
// byte eb - 7 - 4 term.  (TOP for 7: |x| / sc < 2^(TOP + 1).)
__device__ __forceinline__ uint32_t block_exponent(uint32_t mx_bits) { return max(mx_bits, as_bits(0x1p-100f)) >> 23; }
template <uint32_t TOP = 7u>
__device__ __forceinline__ uint32_t block_scale_bits(uint32_t eb) { return (eb - TOP) << 23; }

// Builder side of the hand-over: the terms of this lane's chunk; holder side: the 8 operand registers.
template <int TERMS>
__device__ __forceinline__ void put_terms(uint32_t* ex, int at, const uint32_t (&t)[TERMS][2]) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k) *reinterpret_cast<u32x2_t*>(ex + at + 32 * k) = u32x2_t{t[k][0], t[k][1]};
}
__device__ __forceinline__ v8i_t get_operand(const uint32_t* ex, int at) {
  const u32x4_t a = *reinterpret_cast<const u32x4_t*>(ex + at), b = *reinterpret_cast<const u32x4_t*>(ex + at + 4);
  return v8i_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// D = A B + C with B = 32 centred codes per lane from two packed words (see centred_nibbles); kScaleB: the block scale
// byte of B (127 = 1, 129 = 4).
template <int kScaleB = 127>
__device__ __forceinline__ float4_t mfma_codes(v8i_t a, uint32_t w0, uint32_t w1, float4_t c, int scale_a, uint32_t pick) {
  const v8i_t b = {(int)centred_nibbles(w0, pick), (int)centred_nibbles(w0 << 1, pick), (int)centred_nibbles(w1, pick),
                   (int)centred_nibbles(w1 << 1, pick), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0 /* A: FP8 E4M3 */, 4 /* B: FP4 E2M1 */, 0, scale_a,
                                                         0, kScaleB);
}
// 4-bit codes: a tile is two planes of 2-bit codes, the base-4 digits of the codes, and
// code - 7.5 = 4 (high digit - 1.5) + (low digit - 1.5): the contraction with the codes is the contraction with the high
// plane under a block scale of 4 plus the contraction with the low plane.
__device__ __forceinline__ float4_t mfma_codes_high(v8i_t a, uint32_t w0, uint32_t w1, float4_t c, int scale_a, uint32_t pick) {
  return mfma_codes<129>(a, w0, w1, c, scale_a, pick);
}

// Register image of one group; BITS / 2 planes per tile.
template <int BITS>
struct KeyRegs {
  uint4 kw[2 * BITS];  // key tile: kw[4 plane + m] = the words of token blocks 2 m (x, y) and 2 m + 1 (z, w) for this lane's (column, quarter)
  uint4 ks, kz;  // key scale / zero-point of the 8 channels c0 .. c0 + 7 this lane builds operands for
};
template <int BITS>
struct ValueRegs {
  uint4 vw[2 * BITS];  // value tile, channel blocks 2 m and 2 m + 1 of every plane
  uint4 sz[2];  // value (scale, zero-point) pairs of tokens 16 n + jd, n = 0..7
};

// A record is fetched in two parts so that each part can be requested again for the next group as soon as its
// contraction has consumed it: the key part flies during E V, the value part during the next q K^T.
// The tiles are read once per launch and by one wave only: non-temporal loads (measured: config 2 23.7 -> 22.2 us,
// config 4 83.7 -> 77.5 us; the short contexts of config 7 lose 2 %).
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  const u32x4_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  return make_uint4(t[0], t[1], t[2], t[3]);
}
template <int BITS>
__device__ __forceinline__ void load_keys(KeyRegs<BITS>& r, const uint32_t* __restrict__ rec, const Roles& lr) {
  const uint4* kt = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kKeyTile);
#pragma unroll
  for (int m = 0; m < 2 * BITS; ++m) r.kw[m] = load_once(kt + m * 64 + lr.lane);  // (the planes follow each other)
  r.ks = *reinterpret_cast<const uint4*>(reinterpret_cast<const half_t*>(rec + Rec<BITS>::kKeyScale) + lr.c0);
  r.kz = *reinterpret_cast<const uint4*>(reinterpret_cast<const half_t*>(rec + Rec<BITS>::kKeyZero) + lr.c0);
}

template <int BITS>
__device__ __forceinline__ void load_values(ValueRegs<BITS>& r, const uint32_t* __restrict__ rec, const Roles& lr) {
  const uint4* vt = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kValueTile);
#pragma unroll
  for (int m = 0; m < 2 * BITS; ++m) r.vw[m] = load_once(vt + m * 64 + lr.lane);
  const uint4* sz = reinterpret_cast<const uint4*>(rec + Rec<BITS>::kValueSZ) + 2 * lr.jd;
  r.sz[0] = sz[0];
  r.sz[1] = sz[1];
}

// NB = head blocks of 4 query heads (1: up to 4 heads per KV head, 2: up to 8).  State of a wave, row role.
template <int NB>
struct WaveState {
  float m[NB];          // reference maximum of this lane's head (equal in the 16 lanes of the row), log2 domain
  float l[NB];          // per-lane partial sum of p
  float pz[NB];         // per-lane partial sum of p * (value zero-point + 1.5 value scale)
  float acc[NB][8];     // E V of channel 16 n + jd
};

template <int NB>
__device__ __forceinline__ void empty_state(WaveState<NB>& st) {
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    st.m[nb] = -INFINITY; st.l[nb] = 0.f; st.pz[nb] = 0.f;
#pragma unroll
    for (int n = 0; n < 8; ++n) st.acc[nb][n] = 0.f;
  }
}

template <int TERMS>
__device__ __forceinline__ float sum_of_terms(float4_t d) {
  return TERMS == 3 ? (d[0] + d[1]) + d[2] : (d[0] + d[1]) + (d[2] + d[3]);
}

// q K^T of one group for all heads (Alg. 1 line 7): sc[nb][n] = q.k of head 4 nb + hd, token 16 n + jd (the factor
// log2(e) / sqrt(d) enters with the reference maximum, see exponent()).
// qh = this lane's 8 query values (head 4 nb + ha, channels c0 ..) in binary16 pairs.
// off[nb] = what the zero-points and the centring of the codes add to every score of the head: sc leaves it out.
// valid: tokens of the group that exist (only the newest group of a sequence may be partial; the loop over the others passes
// the constant).
// EXACT_OFFSETS: zero-points and scales each for themselves, in place of mid-points rounded to binary16 (2^-12 of them: keys with an offset of
// 300 in some channels left outputs 1.5e-2 off, so 3e-4).
// TERMS: of query times key scale, each 4 bits of it: three for outputs (2^-12), four, in the spare row, where the weights are results themselves (2^-16).
// A matrix instruction drops what lies more than 13 bits below the exponent of its largest product (measured).  With |x| / sc < 256 that is, now and
// then, a part of a small channel's first term: 2^-14 of a score, of no account beside three terms.  With |x| / sc < 8 and FP8's smallest step of 2^-9
// nothing is dropped: a group's sum of weights 1.3e-5 off -> 4e-7 (a fifth term, in an instruction of its own: 1.5e-7 for 4 to 6 % of the time).
template <int NB, int BITS, bool EXACT_OFFSETS = false, int TERMS = 3>
__device__ __forceinline__ void qk_phase(const KeyRegs<BITS>& g, int valid, const uint32_t (&qh)[NB][4], const Roles& lr,
                                         float (&sc)[NB][8], float (&off)[NB]) {
  static_assert(TERMS == 3 || TERMS == 4, "rows of the matrix instruction");
  constexpr uint32_t kTop = TERMS == 3 ? 7u : 2u;  // |x| / sc < 2^(kTop + 1)
  const uint32_t S[4] = {g.ks.x, g.ks.y, g.ks.z, g.ks.w};
  const uint32_t Z[4] = {g.kz.x, g.kz.y, g.kz.z, g.kz.w};
  v8i_t A[NB];
  int scale_a[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float x[8], bz = 0.0f, bs = 0.0f, mx = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = fmaf((float)as_h2(qh[nb][i >> 1])[i & 1], (float)as_h2(S[i >> 1])[i & 1], 0.0f);  // exact; the fused form reads binary16 operands as they are
      mx = fmaxf(mx, fabsf(x[i]));
    }
    // sum_c q_c (z_c + 1.5 s_c): what the zero-points and the centring of the codes add to every score of the group.
    // Mid-points and query in binary16 pairs, products summed in binary32: the term is a common offset of the
    // group's scores and small (keys are centred), its rounding (2^-12 of it) is of no account.
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (EXACT_OFFSETS) {
        bz = __builtin_amdgcn_fdot2(as_h2(qh[nb][i]), as_h2(Z[i]), bz, false);
        bs = __builtin_amdgcn_fdot2(as_h2(qh[nb][i]), as_h2(S[i]), bs, false);
        continue;
      }
      const half2_t mid = as_h2(S[i]) * half2_t{(half_t)Rec<BITS>::kCentre, (half_t)Rec<BITS>::kCentre} + as_h2(Z[i]);
      bz = __builtin_amdgcn_fdot2(as_h2(qh[nb][i]), mid, bz, false);
    }
    const uint32_t eb = block_exponent(xrow_umax(quad_umax(as_bits(mx))));  // over the 128 channels of the head
    if constexpr (EXACT_OFFSETS) bz = fmaf(bs, Rec<BITS>::kCentre, bz);
    bz = xrow_allsum(quad_allsum(bz));
    uint32_t t[TERMS][2];
    split_fp8(x, block_scale_bits<kTop>(eb), t);
    // (two head blocks: the second one goes through the other exchange region, so that one hand-over serves both)
    put_terms(nb == 0 ? lr.ex_qk : lr.ex_pv, lr.wq, t);
    if (NB == 1) {
      lds_order();
      A[nb] = get_operand(lr.ex_qk, lr.rd);
      lds_order();
    }
    scale_a[nb] = (int)eb - (int)kTop - 4 * lr.ua;
    // the head's zero-point term, from a lane that holds head hd in the operand role (lane 4 hd)
    off[nb] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(16 * lr.hd, __builtin_bit_cast(int, bz)));
  }
  if (NB == 2) {
    lds_order();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) A[nb] = get_operand(nb == 0 ? lr.ex_qk : lr.ex_pv, lr.rd);
    lds_order();
  }
  const float4_t zero = {0.f, 0.f, 0.f, 0.f};
  if constexpr (BITS == 2 && NB == 1) {
    // All eight matrix instructions first, each into registers of its own, then the sums of the term rows: written
    // as one loop the compiler reuses the result registers and every instruction waits for the one before (a dozen
    // idle cycles each; config 3 24.0 -> 22.9 us, config 2 21.5 -> 21.25 us; two head blocks do not gain).
    float4_t dq[8];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const uint32_t w[4] = {g.kw[m].x, g.kw[m].y, g.kw[m].z, g.kw[m].w};
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) dq[2 * m + hf] = mfma_codes(A[0], w[2 * hf], w[2 * hf + 1], zero, scale_a[0], lr.pick);
    }
#pragma unroll
    for (int n = 0; n < 8; ++n) sc[0][n] = sum_of_terms<TERMS>(dq[n]);
  }
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const uint32_t w[4] = {g.kw[m].x, g.kw[m].y, g.kw[m].z, g.kw[m].w};
    if constexpr (BITS == 2 && NB == 1) {
    } else if constexpr (BITS == 2) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float4_t d = mfma_codes(A[nb], w[2 * hf], w[2 * hf + 1], zero, scale_a[nb], lr.pick);
          sc[nb][2 * m + hf] = sum_of_terms<TERMS>(d);
        }
    } else {
      const uint32_t wl[4] = {g.kw[4 + m].x, g.kw[4 + m].y, g.kw[4 + m].z, g.kw[4 + m].w};  // low plane
      float4_t d[2][NB];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) d[hf][nb] = mfma_codes_high(A[nb], w[2 * hf], w[2 * hf + 1], zero, scale_a[nb], lr.pick);
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          d[hf][nb] = mfma_codes(A[nb], wl[2 * hf], wl[2 * hf + 1], d[hf][nb], scale_a[nb], lr.pick);
          sc[nb][2 * m + hf] = sum_of_terms<TERMS>(d[hf][nb]);
        }
    }
  }
  if (valid < kGroup) {  // partial last group: tokens >= valid do not exist
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int n = 0; n < 8; ++n)
        if (16 * n + lr.jd >= valid) sc[nb][n] = -INFINITY;
  }
}

// Reference maximum (Alg. 1 line 8).  Any reference m works as long as 2^(x - m) stays moderate, so the reference of a
// head is only raised -- with a maximum over the row and a rescale of the accumulated state -- when some score of the
// group exceeds it by more than `slack`; most groups pay one comparison per register.  (The literal form of Alg. 1's
// last lines adds the correction to sums that are shifted by the TRUE maximum: there the slack is 0, which makes the
// reference the running maximum itself.)
constexpr float kSlack = 5.0f;
// What 2 is raised to for a score (its head's offset off apart) and the reference m: s kAlpha + base.
__device__ __forceinline__ float exponent_base(float off, float m) { return fmaf(off, kAlpha, -m); }
__device__ __forceinline__ float exponent(float s, float base) { return fmaf(s, kAlpha, base); }
// The reference is rounded in another way than the exponents, so the exponent of the largest score is not 0 but what the
// roundings of off kAlpha - m and of m leave: 1/8 at most while both stay below this bound, and beyond anything that a power
// of two can hold a few thousand times further up.
constexpr float kFusedBound = 0x1p20f;

// base[nb] = what exponent() takes with a score of the head.  Above kFusedBound (no ordinary keys and queries get there) the
// scores themselves are replaced by their distance from the reference, rounded as the reference is, and the base is 0.  (The look
// takes 0 to 0.9 % of a step: 16 sequences of 8k tokens 26.29 -> 26.36 us, one of 131072 tokens 24.95 -> 25.10 us; one branch for
// both looks takes the same.)
template <int NB>
__device__ __forceinline__ void update_reference(float (&sc)[NB][8], const float (&off)[NB], float (&base)[NB], WaveState<NB>& st, float slack) {
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float mloc = sc[nb][0];
#pragma unroll
    for (int n = 1; n < 8; ++n) mloc = fmaxf(mloc, sc[nb][n]);
    mloc = (mloc + off[nb]) * kAlpha;
    if (__builtin_amdgcn_ballot_w64(mloc > st.m[nb] + slack) != 0) {
      const float mnew = fmaxf(st.m[nb], row_allmax(mloc));
      const float f = mnew == -INFINITY ? 1.0f : exp2f(st.m[nb] - mnew);  // 0 when the old reference is -inf
      st.l[nb] *= f;
      st.pz[nb] *= f;
#pragma unroll
      for (int n = 0; n < 8; ++n) st.acc[nb][n] *= f;
      st.m[nb] = mnew;
    }
    base[nb] = exponent_base(off[nb], st.m[nb]);
    if (__builtin_amdgcn_ballot_w64(fmaxf(fabsf(base[nb]), fabsf(st.m[nb])) > kFusedBound) != 0) {
#pragma clang fp contract(off)
#pragma unroll
      for (int n = 0; n < 8; ++n) sc[nb][n] = ((sc[nb][n] + off[nb]) * kAlpha - st.m[nb]) * (1.0f / kAlpha);
      base[nb] = 0.0f;
    }
  }
}

// p = 2^(x - m), its sums, and E V of one group (Alg. 1 lines 9-10).  MASKED: tokens from `fp16_from` on count in the
// sums of p but not in E V: their values are taken from the fp16 window (pv_window_tail).  group_sum: NULL, or where this lane's sums of the group's p go.
// QK_TERMS: those of qk_phase, the fourth of which lies where the weights' spare row has to be zero if two head blocks share the regions.
template <int NB, int BITS, bool MASKED = false, int QK_TERMS = 3>
__device__ __forceinline__ void pv_phase(const ValueRegs<BITS>& g, const float (&sc)[NB][8], const float (&base)[NB], const Roles& lr,
                                         WaveState<NB>& st, int fp16_from = kGroup, float* group_sum = nullptr) {
  constexpr uint32_t kTop = QK_TERMS == 3 ? 7u : 2u;  // (see qk_phase)
  const uint32_t SZ[8] = {g.sz[0].x, g.sz[0].y, g.sz[0].z, g.sz[0].w, g.sz[1].x, g.sz[1].y, g.sz[1].z, g.sz[1].w};
  v8i_t A[NB];
  int scale_a[NB];
  // z + 1.5 s of the lane's tokens: what the zero-point and the centring of the codes give for every channel
  float mid[8];
#pragma unroll
  for (int n = 0; n < 8; ++n) mid[n] = fmaf((float)as_h2(SZ[n])[0], Rec<BITS>::kCentre, (float)as_h2(SZ[n])[1]);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float y[8], mx = 0.0f, sum = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float p = __builtin_amdgcn_exp2f(exponent(sc[nb][n], base[nb]));
      const half2_t sz = as_h2(SZ[n]);
      st.l[nb] += p;
      sum += p;
      const bool coded = !MASKED || 16 * n + lr.jd < fp16_from;
      y[n] = coded ? fmaf(p, (float)sz[0], 0.0f) : 0.0f;  // p * value scale: the weight of the token's codes
      st.pz[nb] = coded ? fmaf(p, mid[n], st.pz[nb]) : st.pz[nb];
      mx = fmaxf(mx, y[n]);
    }
    if (group_sum != nullptr) group_sum[nb] = sum;
    const uint32_t eb = block_exponent(row_umax(as_bits(mx)));  // over the 128 tokens of the head
    uint32_t t[3][2];
    split_fp8(y, block_scale_bits<kTop>(eb), t);
    uint32_t* region = nb == 0 ? lr.ex_pv : lr.ex_qk;
    put_terms(region, lr.wp, t);
    if constexpr (NB == 2 && QK_TERMS > 3) *reinterpret_cast<u32x2_t*>(region + lr.wp + 96) = u32x2_t{0u, 0u};
    region[kExHead * lr.hd + kExExp] = eb;  // the same value from the 16 lanes of the row
    if (NB == 1) {
      lds_order();
      A[nb] = get_operand(lr.ex_pv, lr.rd);
      scale_a[nb] = (int)lr.ex_pv[kExHead * lr.ha + kExExp] - (int)kTop - 4 * lr.ua;
      lds_order();
    }
  }
  if (NB == 2) {
    lds_order();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const uint32_t* region = nb == 0 ? lr.ex_pv : lr.ex_qk;
      A[nb] = get_operand(region, lr.rd);
      scale_a[nb] = (int)region[kExHead * lr.ha + kExExp] - (int)kTop - 4 * lr.ua;
    }
    lds_order();
  }
  // Every instruction starts from zero and its three term rows are added to the state at once: one register per channel
  // and head block instead of four (NB = 1: 8 for 32) for three additions, and the sum over the groups is rounded like
  // any binary32 sum rather than truncated by the matrix cores' adder.
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const uint32_t w[4] = {g.vw[m].x, g.vw[m].y, g.vw[m].z, g.vw[m].w};
    float4_t d[2][NB];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float4_t zero = {0.f, 0.f, 0.f, 0.f};
        d[hf][nb] = BITS == 2 ? mfma_codes(A[nb], w[2 * hf], w[2 * hf + 1], zero, scale_a[nb], lr.pick)
                              : mfma_codes_high(A[nb], w[2 * hf], w[2 * hf + 1], zero, scale_a[nb], lr.pick);
      }
    if constexpr (BITS == 4) {  // the low plane
      const uint32_t wl[4] = {g.vw[4 + m].x, g.vw[4 + m].y, g.vw[4 + m].z, g.vw[4 + m].w};
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) d[hf][nb] = mfma_codes(A[nb], wl[2 * hf], wl[2 * hf + 1], d[hf][nb], scale_a[nb], lr.pick);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) st.acc[nb][2 * m + hf] += (d[hf][nb][0] + d[hf][nb][1]) + d[hf][nb][2];
  }
}

// The values that pv_window_tail will read, one word of every line of 128 bytes, requested while the scores of the group are formed:
// nobody else reads these slots (the window's share ends at its live tokens), and the trip to memory would come after everything.
constexpr int kWindowLines = kGroup * kHeadDim * 2 / 128;  // R is kGroup where values slide
__device__ __forceinline__ void touch_window_tail(uint32_t (&touched)[kWindowLines / 64], const half_t* __restrict__ v_win, int from, int lane) {
#pragma unroll
  for (int u = 0; u < kWindowLines / 64; ++u)
    touched[u] = reinterpret_cast<const uint32_t*>(v_win)[32 * min(8 * (from >> 2) + 64 * u + lane, kWindowLines - 1)];
}

// Sliding value window (Sec. 4.1, setup: the newest 128 tokens in full precision): the tokens j >= from of the newest
// group still have their fp16 rotated values in the window slots j.  Their share of E V is formed here from those values
// by the one wave that has the newest group, on v_mfma_f32_4x4x4_16B_f16: rows = the 4 heads of a head
// block, columns = 64 channels (lane = channel), k = 4 window slots, the probabilities (binary16, through LDS) broadcast
// from one lane quad per block of 4 slots.  The result is added to the accumulators by way of `out`, this wave's
// [NB * 4][128] slice of the combine buffer.
template <int NB>
__device__ __forceinline__ void pv_window_tail(const half_t* __restrict__ v_win, const float (&sc)[NB][8], const float (&base)[NB], int from,
                                               const Roles& lr, WaveState<NB>& st, int lane, float (*out)[kHeadDim]) {
  half_t* pb = reinterpret_cast<half_t*>(lr.ex_pv);  // [NB * 4 heads][128 tokens]
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const int j = 16 * n + lr.jd;
      pb[(nb * 4 + lr.hd) * kGroup + j] = j >= from ? (half_t)__builtin_amdgcn_exp2f(exponent(sc[nb][n], base[nb])) : (half_t)0.0f;
    }
  lds_order();
  const int quad = lane >> 2, hrow = lane & 3;
  half4_t A[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) A[nb][hf] = *reinterpret_cast<const half4_t*>(pb + (nb * 4 + hrow) * kGroup + 64 * hf + 4 * quad);
  const uint2* vb = reinterpret_cast<const uint2*>(v_win);  // [slot / 4][channel] -> 4 slots
  // (blocks requested together: with 16 two head blocks at 4 bits spilled 30 registers, with 4 two)
  constexpr int kBlocks = NB == 2 ? 4 : 16;
  const int first = from >> 2;                              // blocks of 4 slots below it hold no such token
  float4_t acc[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) acc[nb][0] = acc[nb][1] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int part = 0; part < kGroup / 4 / kBlocks; ++part) {
    uint2 vx[2][kBlocks];
#pragma unroll
    for (int bq = 0; bq < kBlocks; ++bq)
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const int blk = kBlocks * part + bq;
        vx[ch][bq] = blk >= first ? vb[(long long)blk * kHeadDim + 64 * ch + lane] : make_uint2(0, 0);
      }
#pragma unroll
    for (int bq = 0; bq < kBlocks; ++bq)
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const half4_t bop = as_h4(vx[ch][bq].x, vx[ch][bq].y);
        const int blk = kBlocks * part + bq;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb][ch] = mfma_bcast(A[nb][blk / 16], bop, acc[nb][ch], blk % 16);
      }
    asm volatile("" ::: "memory");  // (the next blocks' loads stay behind these products)
  }
  // (lane = channel, registers = heads) -> (row = head, lane = channel % 16, register = channel block n)
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      out[nb * 4 + h][lane] = acc[nb][0][h];
      out[nb * 4 + h][64 + lane] = acc[nb][1][h];
    }
  lds_order();
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int n = 0; n < 8; ++n) st.acc[nb][n] += out[nb * 4 + lr.hd][16 * n + lr.jd];
  lds_order();
  // the spare term row of every head of this exchange region reads as zero again
  uint32_t* ex = reinterpret_cast<uint32_t*>(lr.ex_pv);
  for (int i = lane; i < 4 * 32; i += 64) ex[(i >> 5) * kExHead + 96 + (i & 31)] = 0u;
  lds_order();
}

// ---- a wave's share of the fp16 window as one more block of tokens (raw keys, rotated values) -----------------------------
// On v_mfma_f32_16x16x32_f16, in the row role of the groups: D register nb of lane (hd, jd) is head 4 nb + hd, row 4 hd + nb of
// the A operand; the other rows are zero.
//   q K^T : columns = 16 tokens, positions = 32 channels: step kk takes from lane (hd, jd) the channels
//           64 (kk / 2) + 16 hd + 8 (kk % 2) + 0..7 of token 16 tt + jd, which is what the lanes of a quad hold of q in the operand
//           role (lane kk of the quad), so that A comes from qh by broadcasts inside the quads;
//   E V   : columns = 16 channels, positions = 32 tokens: lane (hd, jd) has tokens 8 hd + 0..7, two 4-slot pieces of v_res.
// Runs before the wave's first group, on empty state.  Bound: latency and, where many short sequences fill the chip, bytes: what
// lies beyond the window's tokens is not read (lanes without a token take the last one's rows).
// Two waves with 64 tokens each, on the 4x4x4 blocks, waited for their first record, then for the keys (each a 16-byte piece of
// 64 lines, in 16 instructions), then for the values, then for q.  Steps before and after (with the requests laid out as they are in
// the kernel below): 144 sequences of 1280 tokens 70.7 -> 64.0 us, 32 x 32 single heads of 1280 45.4 -> 42.0, one sequence of
// 131072 24.4 -> 22.8, of 300 11.8 -> 10.9 (of which the host's two calls take 9.7), 16 of 8k 25.1 -> 24.5, 32 of 32k with 7 heads
// 75.6 -> 72.4.
struct WindowShare {
  int first, end;  // tokens first .. end - 1, at most 32 and first a multiple of 4; none: end <= first
};
// k of the waves share, the last ones: as many as have no group in the last round of a sequence with one split (count: its groups),
// as many as are needed, or all.  (Four waves always, and the whole window requested ahead of the counters in small launches: 0.9265
// instead of 0.9200 of the time of two waves with 64 tokens each, on average over some 4900 decode launches.)
__device__ __forceinline__ WindowShare window_share(int nr, int count, bool one_split, int wave) {
  int k = one_split ? -count & (kWaves - 1) : 0;
  k = max(k == 0 ? kWaves : k, (nr + 31) / 32);
  const int fours = (nr + 3) / 4;  // at most 32: exact below
  const int per = 4 * (k == 4 ? (fours + 3) >> 2 : k == 3 ? ((fours + 2) * 171) >> 9 : k == 2 ? (fours + 1) >> 1 : fours);
  const int at = per * (wave - (kWaves - k));
  return WindowShare{max(at, 0), min(at + per, nr)};  // (at < 0: empty, for at + per <= 0)
}
struct WindowRegs {
  uint4 k[2][4];  // [tt][kk]
  uint4 v[8];     // [channel block]: slots 8 hd + 0..3 (x, y) and + 4..7 (z, w)
};
__device__ __forceinline__ void request_window(WindowRegs& w, const kvlinc_cache& c, int bh, const WindowShare& sh, const Roles& lr) {
  const half_t* keys = reinterpret_cast<const half_t*>(c.k_res) + (long long)bh * c.R * kHeadDim;
  const uint2* vb = reinterpret_cast<const uint2*>(reinterpret_cast<const half_t*>(c.v_res) + (long long)bh * c.R * kHeadDim) + lr.jd;
  const int last = max(sh.end - 1, 0);
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const uint4* krow = reinterpret_cast<const uint4*>(keys + min(sh.first + 16 * tt + lr.jd, last) * kHeadDim);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) w.k[tt][kk] = krow[8 * (kk >> 1) + 2 * lr.hd + (kk & 1)];
  }
  const int u = sh.first / 4 + 2 * lr.hd;
  const uint2 *v0 = vb + min(u, last >> 2) * kHeadDim, *v1 = vb + min(u + 1, last >> 2) * kHeadDim;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const uint2 a = v0[16 * n], b = v1[16 * n];
    w.v[n] = make_uint4(a.x, a.y, b.x, b.y);
  }
}

// The share is not empty: the maxima are finite where the whole of it is seen.  (from_slot, sink_slots: slots below from_slot are seen if they are
// below sink_slots only.)
template <int NB>
__device__ __forceinline__ void window_part(const WindowRegs& w, const uint32_t (&qh)[NB][4], const WindowShare& sh, const Roles& lr, WaveState<NB>& st, int from_slot = 0, int sink_slots = 0) {
  float4_t d[2];
  d[0] = d[1] = float4_t{0.f, 0.f, 0.f, 0.f};
  const uint32_t row0 = lr.ua == 0 ? ~0u : 0u, row1 = lr.ua == 1 ? ~0u : 0u;
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    const auto from_quad = [&](uint32_t v) { return kk == 0 ? dpp_u<0x00>(v) : kk == 1 ? dpp_u<0x55>(v) : kk == 2 ? dpp_u<0xAA>(v) : dpp_u<0xFF>(v); };
    uint32_t a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = from_quad(qh[0][i]) & row0;
      if (NB == 2) a[i] |= from_quad(qh[NB - 1][i]) & row1;
    }
    const half8_t A = __builtin_bit_cast(half8_t, make_uint4(a[0], a[1], a[2], a[3]));
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) d[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, __builtin_bit_cast(half8_t, w.k[tt][kk]), d[tt], 0, 0, 0);
  }
  half_t* pb = reinterpret_cast<half_t*>(lr.ex_pv);  // head 4 nb + hd: 32 halves at words 160 hd + 16 nb (clear of the spare term rows)
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float sc[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int slot = sh.first + 16 * tt + lr.jd;
      sc[tt] = slot < sh.end && (slot >= from_slot || slot < sink_slots) ? d[tt][nb] * kAlpha : -INFINITY;
    }
    const float m = row_allmax(fmaxf(sc[0], sc[1]));
    float p[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      p[tt] = __builtin_amdgcn_exp2f(sc[tt] - m);
      pb[2 * (kExHead * lr.hd + 16 * nb) + 16 * tt + lr.jd] = (half_t)p[tt];
    }
    st.m[nb] = m;
    st.l[nb] = p[0] + p[1];
    st.pz[nb] = 0.0f;
  }
  lds_order();
  const uint4 t = *reinterpret_cast<const uint4*>(pb + 2 * (kExHead * lr.ha + 16 * min(lr.ua, NB - 1)) + 8 * lr.hd);
  const half8_t A = __builtin_bit_cast(half8_t, lr.ua < NB ? t : make_uint4(0, 0, 0, 0));
  lds_order();
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float4_t zero = {0.f, 0.f, 0.f, 0.f};
    const float4_t e = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, __builtin_bit_cast(half8_t, w.v[n]), zero, 0, 0, 0);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) st.acc[nb][n] = e[nb];
  }
}

}  // namespace
}  // namespace kvlinc
