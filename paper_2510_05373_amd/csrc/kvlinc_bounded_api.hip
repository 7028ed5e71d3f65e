// Host side of kvlinc_bounded.h: argument validation, workspaces and launch set-up.  Nothing here touches device memory.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kvlinc_bounded_internal.h"
#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

inline bool bad_address(const void* p, uintptr_t a) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

struct Span {
  const void* at;
  unsigned __int128 bytes;
};
bool overlap(const Span& p, const Span& q) {
  const unsigned __int128 a = reinterpret_cast<uintptr_t>(p.at), b = reinterpret_cast<uintptr_t>(q.at);
  return p.at != nullptr && q.at != nullptr && a < b + q.bytes && b < a + p.bytes;
}

long long pairs_of(const kvlinc_cache& c) { return (long long)c.B * c.H_kv; }
// Positions below 2^31, the grids' threads below 2^32.
bool too_large(const kvlinc_cache& c) {
  return pairs_of(c) >= (1ll << 24) || c.max_groups * kGroup + c.R > INT32_MAX - 2 * kGroup || pairs_of(c) * (c.max_groups + 1) >= (1ll << 26);
}
int check_mass_cache(const kvlinc_cache* c) {
  const int rc = kvlinc_cache_validate(c);
  if (rc != KVLINC_OK) return rc;
  return c->S16 != nullptr || too_large(*c) ? KVLINC_EINVAL : KVLINC_OK;
}
size_t mass_bytes(const kvlinc_cache& c) { return (size_t)(pairs_of(c) * (c.max_groups + 1)) * sizeof(float); }
// mass and mass_out of one call over one cache.
bool bad_mass(const kvlinc_cache& c, const float* mass, float decay, const float* mass_out) {
  if (misaligned(mass, 4) || bad_address(mass_out, 4) || !(decay >= 0.0f && decay <= 1.0f)) return true;
  return mass != mass_out && overlap({mass, mass_bytes(c)}, {mass_out, mass_bytes(c)});
}
bool bad_workspace(const void* workspace, size_t bytes, size_t need) { return bad_address(workspace, 16) || bytes < need; }

long long tokens_of_bound(const kvlinc_cache& c, int max_context) {
  const long long cap = c.max_groups * kGroup + c.R;
  return max_context > 0 && max_context < cap ? max_context : cap;
}
long long groups_of_bound(const kvlinc_cache& c, int max_context) {
  const long long groups = (tokens_of_bound(c, max_context) + kGroup - 1) / kGroup;
  return groups < c.max_groups ? groups : c.max_groups;
}

// Decode: two workgroups of four waves a compute unit, as many as have a group for each wave, which the sequences share (part_of in kvlinc_decode_mass.hip).
// Not more than that: from B H_kv = 512 on every pair has one, whatever its length (64 sequences of 8 KV heads: equal lengths of 9216 tokens 65 us, 2k to 16k,
// 1.1 times as many in all, 89; one of 32768 among 500s 110, where 31 of these leave room to share 21); and a pair has kMaxContextSplits at most (one
// sequence of 131072 tokens: 2 KV heads 36 us, 8 of them 33).
struct DecodePlan {
  long long units, slots;
  size_t part_floats, sums;
  size_t bytes() const { return part_floats * sizeof(float) + sums * sizeof(unsigned long long); }
};
DecodePlan plan_decode(const kvlinc_cache& c, int max_context) {
  const long long groups = groups_of_bound(c, max_context), splits = (groups + 3) / 4;
  DecodePlan p{};
  const long long most = c.B * (splits < kMaxContextSplits ? splits : kMaxContextSplits);
  p.units = 512 / c.H_kv;
  if (p.units > most) p.units = most;
  if (p.units < c.B) p.units = c.B;
  p.slots = c.max_groups + 4;  // (the window's 128 tokens in runs of 32; whatever max_context says, so that no sequence is too long for it)
  p.part_floats = p.units > c.B ? (size_t)(p.units * c.H_q) * kPartStride : 0;
  p.sums = (size_t)(pairs_of(c) * p.slots) * 8;
  return p;
}

bool bad_rows(const kvlinc_cache& c, int T) {
  const long long rows = (long long)T * (c.H_q / c.H_kv);
  return T < 1 || T > (1 << 20) || pairs_of(c) * ((rows + 63) / 64) >= (1ll << 22);
}
struct RowsPlan {
  long long slots, rows;
  size_t lse, row_lse;
  size_t bytes() const { return (lse + row_lse) * sizeof(float); }
};
RowsPlan plan_rows(const kvlinc_cache& c, int T, int max_context) {
  RowsPlan p{};
  p.slots = groups_of_bound(c, max_context) + 1;
  p.rows = ((long long)T * (c.H_q / c.H_kv) + 15) / 16 * 16;
  p.lse = (size_t)(pairs_of(c) * p.slots) * (size_t)p.rows;
  p.row_lse = (size_t)(pairs_of(c) * p.rows);
  return p;
}

MassCall make_mass(const kvlinc_cache& c, const kvlinc_half* q, const float* mass, float decay, float* mass_out) {
  MassCall a{};
  a.cache = c;
  a.q = reinterpret_cast<const _Float16*>(q);
  a.mass = decay != 0.0f ? mass : nullptr;
  a.mass_out = mass_out;
  a.decay = decay;
  a.gq = c.H_q / c.H_kv;
  return a;
}

// ---- eviction ----
size_t evict_words(const kvlinc_cache& c) { return evicts_in_one_launch(c) ? 4 : (size_t)(pairs_of(c) * (c.max_groups + 2)); }
constexpr int kBuffers = 5;  // those of a cache that eviction writes
void buffers_of(const kvlinc_cache& c, Span (&s)[kBuffers]) {
  const size_t pairs = (size_t)pairs_of(c), window = pairs * c.R * kHeadDim * 2;
  s[0] = {c.groups, (unsigned __int128)pairs * c.max_groups * (size_t)(c.bits == 2 ? Rec<2>::kWords : Rec<4>::kWords) * 4};
  s[1] = {c.k_res, window};
  s[2] = {c.v_res, window};
  s[3] = {c.n_quant, (size_t)c.B * 4};
  s[4] = {c.n_res, (size_t)c.B * 4};
}

// ---- positions ----
int size_of(int dtype) { return dtype == KVLINC_F32 ? 4 : 2; }
// Memory between the first and the last row of a tensor's input.
Span input_span(const kvlinc_rows& r, const kvlinc_cache& c, int heads, int T, int size) {
  const unsigned __int128 last = (unsigned __int128)r.sequence_stride * (c.B - 1) + (unsigned __int128)r.head_stride * (heads - 1) + (unsigned __int128)r.token_stride * (T - 1);
  return {r.in, (last + kHeadDim) * size};
}

}  // namespace
}  // namespace kvlinc

using namespace kvlinc;

extern "C" {

int kvlinc_rotary(const kvlinc_cache* cache, const kvlinc_rotation* rotation, const kvlinc_rows* q, const kvlinc_rows* k, const kvlinc_rows* v,
                  int32_t T, const int32_t* n_new, const int32_t* first, const int32_t* depth, int32_t counted, int32_t dtype_in,
                  int32_t dtype_out, void* stream) {
  const int rc = kvlinc_cache_validate(cache);
  if (rc != KVLINC_OK) return rc;
  if (rotation == nullptr || rotation->channels < 2 || rotation->channels > kHeadDim || rotation->channels % 2 != 0) return KVLINC_EINVAL;
  if (rotation->interleaved < 0 || rotation->interleaved > 1 || !std::isfinite(rotation->magnitude) || bad_address(rotation->freq, 16)) return KVLINC_EINVAL;
  // (2^26 tokens, four to a workgroup of 256, would be 2^32 threads)
  if (T < 1 || T > (1 << 24) || (long long)cache->B * T > (1ll << 26) - 4 || counted < 0 || counted > 1) return KVLINC_EINVAL;
  if (misaligned(n_new, 4) || misaligned(first, 4) || misaligned(depth, 4)) return KVLINC_EINVAL;
  if (dtype_in < KVLINC_F16 || dtype_in > KVLINC_F32 || dtype_out < KVLINC_F16 || dtype_out > KVLINC_F32) return KVLINC_EINVAL;
  RotaryCall a{};
  const kvlinc_rows* tensors[3] = {q, k, v};
  Span in[3] = {}, out[3] = {};
  for (int i = 0; i < 3; ++i) {
    if (tensors[i] == nullptr) continue;
    const kvlinc_rows& r = *tensors[i];
    const int heads = i == 0 ? cache->H_q : cache->H_kv, aligned = 16 / size_of(dtype_in);
    if (bad_address(r.in, 16) || bad_address(r.out, 16)) return KVLINC_EINVAL;
    for (const int64_t s : {r.sequence_stride, r.head_stride, r.token_stride})
      if (s < 0 || s > (1ll << 48) || s % aligned != 0) return KVLINC_EINVAL;
    in[i] = input_span(r, *cache, heads, T, size_of(dtype_in));
    out[i] = {r.out, (unsigned __int128)cache->B * heads * T * kHeadDim * size_of(dtype_out)};
    a.rows[i] = RotaryRows{r.in, r.out, r.sequence_stride, r.head_stride, r.token_stride, heads};
    a.heads += heads;
  }
  if (a.heads == 0) return KVLINC_EINVAL;
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 3; ++j) {
      if (i < j && overlap(out[i], out[j])) return KVLINC_EINVAL;
      if (!overlap(out[i], in[j])) continue;
      const kvlinc_rows& r = *tensors[j];
      const int64_t heads = j == 0 ? cache->H_q : cache->H_kv;
      const bool in_place = i == j && r.in == r.out && dtype_in == dtype_out && (T == 1 || r.token_stride == kHeadDim) &&
                            (heads == 1 || r.head_stride == (int64_t)T * kHeadDim) && (cache->B == 1 || r.sequence_stride == heads * T * kHeadDim);
      if (!in_place) return KVLINC_EINVAL;
    }
  a.freq = rotation->freq;
  a.magnitude = rotation->magnitude;
  a.channels = rotation->channels;
  a.n_quant = counted != 0 ? cache->n_quant : nullptr;
  a.n_res = counted != 0 ? cache->n_res : nullptr;
  a.first = first;
  a.depth = depth;
  a.n_new = n_new;
  a.B = cache->B;
  a.T = T;
  return launch_rotary(a, rotation->interleaved != 0, dtype_in, dtype_out, static_cast<hipStream_t>(stream));
}

size_t kvlinc_decode_mass_workspace_bytes(const kvlinc_cache* cache, int32_t max_context) {
  return check_mass_cache(cache) == KVLINC_OK ? plan_decode(*cache, max_context).bytes() : 0;
}

int kvlinc_decode_attention_mass(const kvlinc_cache* cache, const kvlinc_half* q, kvlinc_half* out, const float* mass, float decay, float* mass_out,
                                 void* workspace, size_t workspace_bytes, int32_t max_context, void* stream) {
  const int rc = check_mass_cache(cache);
  if (rc != KVLINC_OK) return rc;
  if (bad_address(q, 16) || bad_address(out, 16) || bad_mass(*cache, mass, decay, mass_out)) return KVLINC_EINVAL;
  const size_t bytes = (size_t)cache->B * cache->H_q * kHeadDim * 2;
  if ((q != out && overlap({out, bytes}, {q, bytes})) || overlap({mass_out, mass_bytes(*cache)}, {q, bytes}) || overlap({mass_out, mass_bytes(*cache)}, {out, bytes}) ||
      overlap({mass, mass_bytes(*cache)}, {out, bytes}))
    return KVLINC_EINVAL;
  const DecodePlan p = plan_decode(*cache, max_context);
  if (bad_workspace(workspace, workspace_bytes, p.bytes())) return KVLINC_EWORKSPACE;
  MassCall a = make_mass(*cache, q, mass, decay, mass_out);
  a.T = 1;
  a.out = reinterpret_cast<_Float16*>(out);
  a.units = (int)p.units;
  a.slots = p.slots;
  a.sums = static_cast<unsigned long long*>(workspace);
  a.part = p.part_floats != 0 ? reinterpret_cast<float*>(a.sums + p.sums) : nullptr;  // (sums: a multiple of 64 bytes)
  return launch_decode_mass(a, static_cast<hipStream_t>(stream));
}

size_t kvlinc_attention_mass_workspace_bytes(const kvlinc_cache* cache, int32_t T, int32_t max_context) {
  return check_mass_cache(cache) == KVLINC_OK && !bad_rows(*cache, T) ? plan_rows(*cache, T, max_context).bytes() : 0;
}

int kvlinc_attention_mass(const kvlinc_cache* cache, const kvlinc_half* q, const int32_t* n_rows, int32_t T, const float* mass, float decay,
                          float* mass_out, void* workspace, size_t workspace_bytes, int32_t max_context, void* stream) {
  const int rc = check_mass_cache(cache);
  if (rc != KVLINC_OK) return rc;
  if (bad_rows(*cache, T) || bad_address(q, 16) || misaligned(n_rows, 4) || bad_mass(*cache, mass, decay, mass_out)) return KVLINC_EINVAL;
  if (overlap({mass_out, mass_bytes(*cache)}, {q, (size_t)cache->B * cache->H_q * T * kHeadDim * 2})) return KVLINC_EINVAL;
  const RowsPlan p = plan_rows(*cache, T, max_context);
  if (bad_workspace(workspace, workspace_bytes, p.bytes())) return KVLINC_EWORKSPACE;
  MassCall a = make_mass(*cache, q, mass, decay, mass_out);
  a.n_rows = n_rows;
  a.T = T;
  a.slots = p.slots;
  a.bound = (int)tokens_of_bound(*cache, max_context);
  a.rows = (int)p.rows;
  a.lse = static_cast<float*>(workspace);
  a.row_lse = a.lse + p.lse;
  return launch_attention_mass(a, static_cast<hipStream_t>(stream));
}

size_t kvlinc_cache_evict_workspace_bytes(const kvlinc_cache* cache) { return check_mass_cache(cache) == KVLINC_OK ? evict_words(*cache) * sizeof(int32_t) : 0; }

int kvlinc_cache_evict(const kvlinc_cache* from, const kvlinc_cache* to, const float* mass, float* mass_out, int32_t keep, int32_t limit,
                       int32_t first, int32_t last, const int32_t* offset, int32_t* offset_out, int32_t* kept, void* workspace,
                       size_t workspace_bytes, void* stream) {
  int rc = check_mass_cache(from);
  if (rc == KVLINC_OK) rc = check_mass_cache(to);
  if (rc != KVLINC_OK) return rc;
  if (from->B != to->B || from->H_q != to->H_q || from->H_kv != to->H_kv || from->R != to->R || from->bits != to->bits || from->flags != to->flags) return KVLINC_EINVAL;
  if (keep < 1 || limit < keep || first < 0 || last < 1 || first > keep || last > keep - first) return KVLINC_EINVAL;
  if (to->max_groups < (limit < from->max_groups ? limit : from->max_groups)) return KVLINC_EINVAL;
  if (bad_address(mass, 4) || bad_address(mass_out, 4) || misaligned(offset, 4) || misaligned(offset_out, 4) || misaligned(kept, 4)) return KVLINC_EINVAL;
  const bool in_place = from->groups == to->groups && from->k_res == to->k_res && from->v_res == to->v_res && from->n_quant == to->n_quant &&
                        from->n_res == to->n_res && from->max_groups == to->max_groups;
  // what is read, and what is written
  Span in[kBuffers + 2], out[kBuffers + 3];
  Span (&in_cache)[kBuffers] = reinterpret_cast<Span (&)[kBuffers]>(in);
  Span (&out_cache)[kBuffers] = reinterpret_cast<Span (&)[kBuffers]>(out);
  buffers_of(*from, in_cache);
  buffers_of(*to, out_cache);
  in[kBuffers] = {mass, mass_bytes(*from)};
  in[kBuffers + 1] = {offset, (size_t)from->B * 4};
  out[kBuffers] = {mass_out, mass_bytes(*to)};
  out[kBuffers + 1] = {offset_out, (size_t)to->B * 4};
  out[kBuffers + 2] = {kept, (unsigned __int128)pairs_of(*to) * to->max_groups * 4};
  for (int i = 0; i < kBuffers + 3; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return KVLINC_EINVAL;
    for (int j = 0; j < kBuffers + 2; ++j) {
      const bool same = i == j && (i < kBuffers ? in_place : i == kBuffers ? mass == mass_out && from->max_groups == to->max_groups : offset == offset_out);
      if (!same && overlap(out[i], in[j])) return KVLINC_EINVAL;
    }
  }
  if (bad_workspace(workspace, workspace_bytes, evict_words(*from) * sizeof(int32_t))) return KVLINC_EWORKSPACE;
  EvictCall a{};
  a.from = *from;
  a.to = *to;
  a.mass = mass;
  a.mass_out = mass_out;
  a.keep = keep; a.limit = limit; a.first = first; a.last = last;
  a.offset = offset;
  a.offset_out = offset_out;
  a.kept = kept;
  a.in_place = in_place;
  a.counted = in_place || mass == mass_out;
  if (!evicts_in_one_launch(*from)) {
    a.stride = from->max_groups;
    a.source = static_cast<int32_t*>(workspace);
    a.count = a.source + pairs_of(*from) * a.stride;
  }
  return launch_evict(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
