"""Prompt attention of channels whose keys and queries differ by many powers of two, one making up for the other: what a channel gives to a score is
held relative to the score's parts, whatever the magnitudes of keys and queries taken alone."""
import numpy as np
import pytest

from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def run(T, bits, key_gain, query_gain, n=400, rows_exact=False):
    """key_gain, query_gain: powers of two of the 128 channels."""
    H_q, H_kv = 4, 1
    K, V, q, k_new, v_new = ref.inputs(1020, 1, H_q, H_kv, [n], T)
    half = lambda x, e: np.clip(x.astype(np.float64) * 2.0 ** e, -65504, 65504).astype(np.float16)
    K, k_new, q = [[half(K[0][0], key_gain)]], half(k_new, key_gain), half(q, query_gain)
    cache = filled(1, H_q, H_kv, K, V, n + 128, bits)
    assert cache.status.item() == 0
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0], bits)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    for h in range(H_q):
        y, tol = ref.attend(q[0, h], keys, values, n + np.arange(T))
        if rows_exact:  # (few rows take keys as they are: no 2^-11 of a key in the scores, binary32 sums only)
            x = q[0, h].astype(np.float64)
            seen = np.arange(len(keys)) <= n + np.arange(T)[:, None]
            s = np.where(seen, x @ keys.T / np.sqrt(128.0), -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            d = 2.0 ** -14 * np.where(seen, np.abs(x) @ np.abs(keys).T, 0.0).max(1) / np.sqrt(128.0)
            tol = ref.HALF_STEP * np.linalg.norm(y, axis=1) + (2 * ref.HALF_STEP + np.expm1(2 * d)) * (w @ np.linalg.norm(values, axis=1))
        ref.check_rows(got[0, h], y, tol, (T, bits, h))


CHANNELS = np.arange(128)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [1, 2, 3, 12, 40, 300])
@pytest.mark.parametrize("spread", [0, 6, 10, 12])
def test_halves_of_the_channels(T, bits, spread):
    # keys 2^spread and 2^-spread, queries the other way round, with scores of a few units either way
    e = np.where(CHANNELS % 2 == 0, spread, -spread)
    run(T, bits, e, -e, rows_exact=T <= 12)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [3, 12, 40, 300])
@pytest.mark.parametrize("key, query", [(-14, 13), (-18, 13), (-20, 13), (-12, 12), (12, -12), (13, -20), (14, -14), (0, -24)])
def test_small_keys_of_large_queries_and_the_other_way_round(T, bits, key, query):
    run(T, bits, np.full(128, key), np.full(128, query), rows_exact=T <= 12)


@pytest.mark.parametrize("T", [3, 12, 40, 300])
@pytest.mark.parametrize("key, query", [(10, -9), (13, -12)])
def test_one_channel_of_large_keys(T, key, query):
    # a channel whose keys are thousands and whose queries are next to nothing, beside channels of ordinary keys and of large queries
    ek, eq = np.zeros(128), np.zeros(128)
    ek[5], eq[5] = key, query
    ek[64:], eq[64:] = -9, 10
    run(T, 2, ek, eq, rows_exact=T <= 12)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [1, 2, 3, 12, 40, 300])
@pytest.mark.parametrize("large, small, window", [(8000.0, 2.0 ** -8, 0), (8000.0, 2.0 ** -8, 150), (1000.0, 2.0 ** -11, 0), (1.0, 1.0, 0)])
def test_large_values_of_tokens_without_weight(T, bits, large, small, window):
    # one token in 40 has values some 2^21 times the others', and keys against all queries: its weight is below e^-30, or it is out of the window
    H_q, H_kv, n = 4, 1, 500
    K, V, q, k_new, v_new = ref.inputs(1021, 1, H_q, H_kv, [n], T)
    rng = np.random.default_rng(7)
    sign = np.where(rng.random(128) < 0.5, -1.0, 1.0)
    q = (2.0 * np.abs(q.astype(np.float64)) * sign).astype(np.float16)
    K, V, v_new = K[0][0].astype(np.float64), V[0][0].astype(np.float64) * small, v_new.astype(np.float64) * small
    at = np.arange(3, n, 40)
    K[at], V[at] = -6.0 * sign, np.clip(V[at] / small, -2, 2) * large
    if large > 1:
        assert (q.astype(np.float64)[0] @ (6.0 * sign)).min() / np.sqrt(128.0) > 35
    K, V, v_new = [[K.astype(np.float16)]], [[V.astype(np.float16)]], v_new.astype(np.float16)
    cache = filled(1, H_q, H_kv, K, V, n + 128, bits)
    assert cache.status.item() == 0
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new), window=window).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0], bits)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    t, p = np.arange(len(keys)), n + np.arange(T)[:, None]
    seen, norms = (t <= p) & ((window == 0) | (p - t < window)), np.linalg.norm(values, axis=1)
    for h in range(H_q):
        y, _ = ref.attend(q[0, h], keys, values, n + np.arange(T), window)
        x = q[0, h].astype(np.float64)
        s = np.where(seen, x @ keys.T / np.sqrt(128.0), -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        # a score's own error, 2^-11 (few rows: no part of it) and binary32's share of its parts (see context_reference), moves its weight, and the
        # weighted mean of all of them the sum
        d = ((2.0 ** -11 if T > 12 else 0.0) + 2.0 ** -14) * (np.abs(x) @ np.abs(keys).T) / np.sqrt(128.0)
        moved = np.expm1(d + (w * d).sum(1, keepdims=True))
        tol = ref.HALF_STEP * np.linalg.norm(y, axis=1) + (w * (2 * ref.HALF_STEP + moved)) @ norms + 128 ** 0.5 * 2.0 ** -25  # (a subnormal output)
        ref.check_rows(got[0, h], y, tol, (T, bits, h))
