// Host side of kvlinc_context.h: argument validation, workspaces and launch set-up.  Nothing here touches device memory.
#include <hip/hip_runtime.h>

#include "kvlinc_context_internal.h"

namespace kvlinc {
namespace {

inline bool bad_address(const void* p, uintptr_t a) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Whether rows [.., 128] of two tensors share memory.
bool overlap(const void* p, long long p_bytes, const void* q, long long q_bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + (uintptr_t)q_bytes && b < a + (uintptr_t)p_bytes;
}

// What a call makes of its sizes: splits of a context, scratch.
struct ContextPlan {
  // 16 rows a wave (kvlinc_rows.hip); blocks of 256 rows over tiles of codes (kvlinc_prompt.hip), or of rows dequantized first (kvlinc_dense.hip)
  enum Kind { kRows, kTiles, kDense } kind;
  int splits, waves;
  long long cached_rows, sink_rows;      // dequantized rows of a (sequence, KV head)
  int row_window;                        // see ContextCall
  size_t corr_floats, part_floats, row_halfs;  // row_halfs: of keys, and as many of values
  size_t low_words() const { return row_halfs / 8; }  // 4 bits each; and 4 bytes a row
  size_t bytes() const {
    return (corr_floats + part_floats + low_words() + row_halfs / kHeadDim) * sizeof(float) + 2 * row_halfs * sizeof(_Float16);
  }
};

// Groups a row of queries meets in a context of the bound.
long long groups_met(const kvlinc_cache& c, int T, int window, int sinks, int max_context) {
  const long long cap = (long long)c.max_groups * kGroup + c.R;
  const long long ctx = max_context > 0 && max_context < cap ? max_context : cap;
  const long long all = (ctx + kGroup - 1) / kGroup;
  if (window == 0) return all;
  const long long near = ((long long)window + T + kGroup - 1) / kGroup + 1 + ((long long)sinks + kGroup - 1) / kGroup;
  return near < all ? near : all;
}

// (The figures beside the choices below are two sides of one run each, three states in turn so that no cache holds them.)
// Which of the three a call of so many rows a KV head takes, measured (us; 8 KV heads, 2 bits):
//   rows                                   64            512            640            1000
//   1 sequence, 32k cached tokens          rows 53       tiles 137      tiles 200      tiles 245
//                                          tiles 66      dense 149      dense 172      dense 213
//   8 sequences of 4k                      rows 34       tiles 137      tiles 239      tiles 246
//                                          tiles 56      dense 151      dense 190      dense 215
// Every block of 256 rows dequantizes the tiles it goes over anew: from the third block on it pays to have done that once for all.  A wave of
// the first kind has 16 rows and the codes for itself alone: 64 rows are what its registers and four waves make of a pair.
constexpr long long kFewRows = 64, kTiledRows = 2 * 256;
ContextPlan plan_call(const kvlinc_cache& c, int T, int window, int sinks, int max_context) {
  const long long rows = (long long)T * (c.H_q / c.H_kv), pairs = (long long)c.B * c.H_kv;
  const long long groups = groups_met(c, T, window, sinks, max_context);
  ContextPlan p{};
  p.kind = rows <= kFewRows ? ContextPlan::kRows : rows <= kTiledRows ? ContextPlan::kTiles : ContextPlan::kDense;
  long long s, most;
  if (p.kind == ContextPlan::kRows) {
    // Two workgroups of four waves a compute unit, or, where the pairs are few, one of eight: fewer splits to join (6 tokens over 131072, 8 pairs:
    // 58.1 us with four, 50.5 with eight; 4 tokens, 64 pairs of 16k: 29.5 and 27.6; 128 of 8k: 29.6 and 28.6, with the correction 32.2 and 41.1; 512 pairs
    // of 400 to 4096: 41 and 46).
    p.waves = pairs <= 64 ? 8 : 4;
    s = (p.waves == 8 ? 256 : 512) / pairs - (c.S16 != nullptr ? 1 : 0);  // (the correction's workgroups are some of them)
    most = (groups + p.waves - 1) / p.waves;
  } else {
    // One workgroup a compute unit.  A split of less than 8 tiles costs more to write and join than it saves (one prompt of 700 tokens: 31 us, 34 in
    // three splits; 300 tokens over 4096: 63 with 8, 4 and 2), one over codes, whose tiles take longer, of less than 4 (64 tokens over 8192: 54 us with 8, 48
    // with 4 and with 2; over 2048, where two would be better still: 47, 37, 34).  (Without a bound the cache is taken to have room for the rows, no more:
    // that is a guess for the number of splits, not for what is reserved.)
    const long long least = p.kind == ContextPlan::kTiles ? 4 : 8;
    const long long cached = max_context > 0 ? groups * kGroup : groups * kGroup - T;
    s = 256 / (pairs * ((rows + 255) / 256));
    most = ((cached < 0 ? 0 : cached) + T / 2) / (least * kTileTokens);  // (causal: half of the rows on average)
  }
  if (s > most) s = most;
  if (s > kMaxContextSplits) s = kMaxContextSplits;
  if (s < 1) s = 1;
  p.splits = (int)s;
  const size_t places = (size_t)c.B * c.H_q * T;
  p.corr_floats = c.S16 != nullptr ? places * kPartStride : 0;
  p.part_floats = s > 1 || (p.kind == ContextPlan::kRows && p.corr_floats != 0) ? places * s * kPartStride : 0;
  if (p.kind == ContextPlan::kDense) {
    // all cached tokens; or those near the first row, and the sinks ahead of them where there can be such
    const long long cap = (long long)c.max_groups * kGroup + c.R, ctx = max_context > 0 && max_context < cap ? max_context : cap;
    const auto up = [](long long n) { return (n + kTileTokens - 1) / kTileTokens * kTileTokens; };
    const long long near = up(window + (long long)kTileTokens);
    p.cached_rows = up(ctx);
    if (window > 0 && near + up(sinks) < p.cached_rows) {
      p.sink_rows = up(sinks);
      p.cached_rows = near + p.sink_rows;
      p.row_window = window;
    }
    p.row_halfs = (size_t)(pairs * p.cached_rows * kHeadDim);
  }
  return p;
}

// The grids of a call stay below 2^32 threads (rows beyond that would not fit any card's memory), positions below 2^31.
bool too_many(const kvlinc_cache& c, int T) {
  const long long gq = c.H_q / c.H_kv;
  return (long long)c.B * c.H_kv >= (1ll << 24) || (long long)c.B * c.H_kv * ((T * gq + 15) / 16) >= (1ll << 24) ||
         c.max_groups * kGroup + c.R + T > INT32_MAX - 2 * kGroup;
}

int check_prompt(const kvlinc_cache* c, int T, int window, int sinks) {
  const int rc = kvlinc_cache_validate(c);
  if (rc != KVLINC_OK) return rc;
  if (T < 1 || T > (1 << 24) || window < 0 || sinks < 0 || too_many(*c, T)) return KVLINC_EINVAL;
  // the states stand for all quantized tokens; the literal form needs the maximum over the whole context at one place
  if (c->S16 != nullptr && (window != 0 || (c->flags & KVLINC_FLAG_ALG1_LITERAL) != 0)) return KVLINC_EINVAL;
  return KVLINC_OK;
}
// Windowed decode: two workgroups of four waves a compute unit; a split has a group for each wave (from a graph: one sequence, window 1024: 7.3 us, 7.1
// with three groups a wave; 2048: 7.6 and 8.9; 4 bits, 7 heads, 2048: 10.8 and 13.3).
ContextPlan plan_windowed(const kvlinc_cache& c, int window, int sinks, int max_context) {
  const long long pairs = (long long)c.B * c.H_kv, groups = groups_met(c, 1, window, sinks, max_context);
  long long s = 512 / pairs, most = (groups + 3) / 4;
  if (s > most) s = most;
  if (s > kMaxContextSplits) s = kMaxContextSplits;
  if (s < 1) s = 1;
  ContextPlan p{};
  p.splits = (int)s;
  p.part_floats = s > 1 ? (size_t)c.B * c.H_q * s * kPartStride : 0;
  return p;
}

int check_windowed(const kvlinc_cache* c, int window, int sinks) {
  const int rc = kvlinc_cache_validate(c);
  if (rc != KVLINC_OK) return rc;
  return window < 0 || sinks < 0 || c->S16 != nullptr || too_many(*c, 1) ? KVLINC_EINVAL : KVLINC_OK;
}

ContextCall make_call(const kvlinc_cache& c, const kvlinc_half* q, int T, int window, int sinks, kvlinc_half* out, void* workspace, const ContextPlan& p) {
  ContextCall a{};
  a.cache = c;
  a.q = reinterpret_cast<const _Float16*>(q);
  a.T = T; a.window = window; a.sinks = window != 0 ? sinks : 0;
  a.gq = c.H_q / c.H_kv;
  a.splits = p.splits;
  a.corr = p.corr_floats != 0 ? static_cast<float*>(workspace) : nullptr;
  a.part = p.part_floats != 0 ? static_cast<float*>(workspace) + p.corr_floats : nullptr;
  if (p.row_halfs != 0) {  // (the parts before are multiples of 16 bytes)
    a.k_rows = reinterpret_cast<_Float16*>(static_cast<float*>(workspace) + p.corr_floats + p.part_floats);
    a.v_rows = a.k_rows + p.row_halfs;
    a.k_low = reinterpret_cast<uint32_t*>(a.v_rows + p.row_halfs);
    a.k_low_scale = a.k_low + p.low_words();
  }
  a.cached_rows = (int)p.cached_rows;
  a.sink_rows = (int)p.sink_rows;
  a.row_window = p.row_window;
  a.out = reinterpret_cast<_Float16*>(out);
  return a;
}
bool bad_workspace(const void* workspace, size_t bytes, size_t need) { return need != 0 && (bad_address(workspace, 16) || bytes < need); }

}  // namespace
}  // namespace kvlinc

using namespace kvlinc;

extern "C" {

size_t kvlinc_prompt_workspace_bytes(const kvlinc_cache* cache, int32_t T, int32_t window, int32_t sinks, int32_t max_context) {
  return check_prompt(cache, T, window, sinks) == KVLINC_OK ? plan_call(*cache, T, window, sinks, max_context).bytes() : 0;
}

int kvlinc_prompt_attention(const kvlinc_cache* cache, const kvlinc_half* q, const kvlinc_half* k_new, const kvlinc_half* v_new,
                            const int32_t* n_new, int32_t T, int32_t window, int32_t sinks, kvlinc_half* out, void* workspace,
                            size_t workspace_bytes, int32_t max_context, void* stream) {
  const int rc = check_prompt(cache, T, window, sinks);
  if (rc != KVLINC_OK) return rc;
  if (bad_address(q, 16) || bad_address(k_new, 16) || bad_address(v_new, 16) || bad_address(out, 16)) return KVLINC_EINVAL;
  if (n_new != nullptr && bad_address(n_new, 4)) return KVLINC_EINVAL;
  const long long q_bytes = (long long)cache->B * cache->H_q * T * kHeadDim * 2, kv_bytes = q_bytes / (cache->H_q / cache->H_kv);
  if (overlap(out, q_bytes, q, q_bytes) || overlap(out, q_bytes, k_new, kv_bytes) || overlap(out, q_bytes, v_new, kv_bytes)) return KVLINC_EINVAL;
  const ContextPlan p = plan_call(*cache, T, window, sinks, max_context);
  if (bad_workspace(workspace, workspace_bytes, p.bytes())) return KVLINC_EWORKSPACE;
  ContextCall a = make_call(*cache, q, T, window, sinks, out, workspace, p);
  a.k_new = reinterpret_cast<const _Float16*>(k_new);
  a.v_new = reinterpret_cast<const _Float16*>(v_new);
  a.n_new = n_new;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.kind == ContextPlan::kRows) return launch_rows(a, p.waves, s);
  if (a.corr != nullptr) {
    const int rl = launch_prompt_correction(a, s);
    if (rl != KVLINC_OK) return rl;
  }
  return p.kind == ContextPlan::kTiles ? launch_tiles(a, s) : launch_dense(a, s);
}

size_t kvlinc_decode_windowed_workspace_bytes(const kvlinc_cache* cache, int32_t window, int32_t sinks, int32_t max_context) {
  return check_windowed(cache, window, sinks) == KVLINC_OK ? plan_windowed(*cache, window, sinks, max_context).bytes() : 0;
}

int kvlinc_decode_attention_windowed(const kvlinc_cache* cache, const kvlinc_half* q, int32_t window, int32_t sinks, kvlinc_half* out,
                                     void* workspace, size_t workspace_bytes, int32_t max_context, void* stream) {
  const int rc = check_windowed(cache, window, sinks);
  if (rc != KVLINC_OK) return rc;
  if (bad_address(q, 16) || bad_address(out, 16)) return KVLINC_EINVAL;
  // (a head's workgroups have all read q when the last of them writes its row)
  const long long bytes = (long long)cache->B * cache->H_q * kHeadDim * 2;
  if (q != out && overlap(out, bytes, q, bytes)) return KVLINC_EINVAL;
  const ContextPlan p = plan_windowed(*cache, window, sinks, max_context);
  if (bad_workspace(workspace, workspace_bytes, p.bytes())) return KVLINC_EWORKSPACE;
  return launch_windowed(make_call(*cache, q, 1, window, sinks, out, workspace, p), static_cast<hipStream_t>(stream));
}

int kvlinc_cache_read(const kvlinc_cache* cache, const int32_t* first, int32_t T, void* k_out, void* v_out, int32_t dtype,
                      int32_t rotated, void* stream) {
  const int rc = kvlinc_cache_validate(cache);
  if (rc != KVLINC_OK) return rc;
  if (T < 1 || T > (1 << 30) || dtype < KVLINC_F16 || dtype > KVLINC_F32 || rotated < 0 || rotated > 1) return KVLINC_EINVAL;
  if (k_out == nullptr && v_out == nullptr) return KVLINC_EINVAL;
  if ((k_out != nullptr && bad_address(k_out, 16)) || (v_out != nullptr && bad_address(v_out, 16))) return KVLINC_EINVAL;
  if (first != nullptr && bad_address(first, 4)) return KVLINC_EINVAL;
  const long long rows = (long long)cache->B * cache->H_kv * T;  // below 2^55
  if (rows > (1ll << 40)) return KVLINC_EINVAL;  // 2^48 bytes: beyond any address space, and below what 64 bits count
  const long long bytes = rows * kHeadDim * (dtype == KVLINC_F32 ? 4 : 2);
  if (k_out != nullptr && v_out != nullptr && overlap(k_out, bytes, v_out, bytes)) return KVLINC_EINVAL;
  return launch_read(*cache, first, T, k_out, v_out, dtype, rotated != 0, static_cast<hipStream_t>(stream));
}

}  // extern "C"
