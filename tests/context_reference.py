"""64-bit reference of the calls of kvlinc_context.h, from the oracle's cache: dequantized tokens, one softmax, visibility by the definition."""
import numpy as np

import kvlinc_synth as synth
from oracle import attention as o_attn
from oracle import hadamard
from oracle import kvcache as o_cache

# Tolerance of an output row (128 numbers y of a softmax with weights w_t and values v_t), by the roundings of the arithmetic:
#   - y itself to binary16: half a step, 2^-11 |y|;
#   - every weight, and every value that is dequantized ahead of its product, to binary16 once: 2^-11 each of w_t |v_t|;
#   - scores: keys that are dequantized ahead of the product, 2^-11 of each |q_c k_c|, so d_t = 2^-11 sum_c |q_c k_c| / sqrt(128) at
#     most; binary32 sums add 2^-24 a term, 128 of them, and reference and exponent a few 2^-24 |s|: below 2^-14 sum |q k| / sqrt(128);
#   - an error d of the scores moves a normalised weight by a factor of e^(2 d) at most.
# The rotation keeps 2-norms, so all of it holds for the row's norm.
HALF_STEP = 2.0 ** -11


def bound_of_rows(y, w, values, qk_abs):
    """Largest 2-norm by which a row of y may be off; w: weights (normalised, without the correction's share), qk_abs: max_t sum_c |q_c k_c|."""
    d = (2.0 ** -11 + 2.0 ** -14) * qk_abs / np.sqrt(128.0)
    spread = w @ np.linalg.norm(values, axis=1)
    return HALF_STEP * np.linalg.norm(y, axis=1) + (2 * HALF_STEP + np.expm1(2 * d)) * spread


def tokens_of(K, V, n_quant, bits=2, sliding=False, Wk=None):
    """(keys, values in the original basis, cache) of the oracle's cache of one (sequence, KV head)."""
    ref = o_cache.build_cache(K, V, n_quant, bits=bits, Wk=Wk)
    if len(K) == 0:
        return np.zeros((0, 128)), np.zeros((0, 128)), ref
    keys, rotated = o_attn._operands(ref, "sliding" if sliding else "block")
    return keys, rotated @ hadamard.orthonormal(128).T, ref


def attend(q, keys, values, positions, window=0, sinks=0, ref=None, Wq=None):
    """Rows q [r, 128] at `positions` over tokens 0 .. len(keys) - 1: (y, bound on the 2-norm of a row's error)."""
    q = np.asarray(q, dtype=np.float64)
    t = np.arange(len(keys))
    p = np.asarray(positions)[:, None]
    seen = t <= p
    if window:
        seen &= (p - t < window) | (t < sinks)
    s = np.where(seen, q @ keys.T / np.sqrt(128.0), -np.inf)
    m = s.max(1, keepdims=True)
    if Wq is not None:
        m = np.maximum(m, 0.0)
    e = np.exp(s - m)
    num, den = e @ values, e.sum(1, keepdims=True)
    if Wq is not None:
        phi = o_cache.feature_map(q, np.asarray(Wq, dtype=np.float64))
        c = np.exp(-m)
        num = num + c * (phi @ ref["S"]) @ hadamard.orthonormal(128).T
        den = den + c * (phi @ ref["P"])[:, None]
    y = num / den
    qk = np.where(seen, np.abs(q) @ np.abs(keys).T, 0.0).max(1)
    b = bound_of_rows(y, e / den, values, qk)
    if Wq is not None:  # features and states to binary16 (the states' own share of an entry's rounding is in the sums), once each
        b += 2 * HALF_STEP * np.exp(-m[:, 0]) / den[:, 0] * (phi @ np.linalg.norm(ref["S"], axis=1))
        b += 2 * HALF_STEP * np.linalg.norm(y, axis=1)  # the features' softmax as weights of the denominator
    return y, b


def inputs(config, B, H_q, H_kv, lengths, T, scale=1.0):
    """Cached keys and values per (b, g) (fp16), then q, k_new, v_new of T rows."""
    K = [[synth.keys(config, b, g, int(lengths[b]) + T) for g in range(H_kv)] for b in range(B)]
    V = [[synth.values(config, b, g, int(lengths[b]) + T) for g in range(H_kv)] for b in range(B)]
    q = np.stack([[synth.queries(config, b, H_q, step=i) for i in range(T)] for b in range(B)]) if T else np.zeros((B, 0, H_q, 128), np.float16)
    q = (q.astype(np.float32) * scale).astype(np.float16)
    q = np.ascontiguousarray(q.transpose(0, 2, 1, 3))
    k_new = np.stack([[K[b][g][int(lengths[b]):] for g in range(H_kv)] for b in range(B)])
    v_new = np.stack([[V[b][g][int(lengths[b]):] for g in range(H_kv)] for b in range(B)])
    K = [[K[b][g][:int(lengths[b])] for g in range(H_kv)] for b in range(B)]
    V = [[V[b][g][:int(lengths[b])] for g in range(H_kv)] for b in range(B)]
    return K, V, q, k_new, v_new


def check_rows(got, want, bound, what):
    """Every row within its bound; what random roundings of that size come to in fact, 2e-3 of all rows together, over several rows."""
    d = np.linalg.norm(got.astype(np.float64) - want, axis=-1)
    assert np.isfinite(got).all(), what
    worst = (d - bound).argmax()
    assert (d <= bound).all(), (what, int(worst), d.flat[worst], np.asarray(bound).flat[worst])
    return float((d ** 2).sum()), float((want ** 2).sum())
