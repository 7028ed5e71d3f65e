"""Prompt attention with adapters where every logit of a row lies far below zero: e^M, M the largest one, leaves the normal range of binary32 at
-87.3 and all of it at -103.3, but a softmax to which nothing is added does not hang on it, nor does one to which the correction adds as little."""
import numpy as np
import pytest

import kvlinc_synth as synth
import paper_2510_05373_amd as kv
from oracle import hadamard
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu

# All keys alike (exact in codes: scale 0), all queries 2: the logits are -128 * 2 / sqrt(128) times these, -9 to -996, without a rounding.
KEYS = [0.390625, 3.5, 3.875, 4.25, 4.875, 44.0]
H_q = 4


def run(n, T, bits, key, P0=None, sliding=False, bound=0):
    """Every row against the closed form; P0: what P holds instead of its sums, with S = 0."""
    K, V, q, k_new, v_new = ref.inputs(89, 1, H_q, 1, [n], T)
    K[0][0][:], q[:], k_new[:] = -key, 2.0, -key
    Wq, Wk = synth.adapters_q(89, H_q), synth.adapters_k(89, 1)
    cache = filled(1, H_q, 1, K, V, n + 128, bits, kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0, to_dev(Wq), to_dev(Wk))
    if P0 is not None:
        cache.S16.zero_()
        cache.P.fill_(P0)
    out = np.asarray(cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new), max_context=bound).cpu().numpy(), dtype=np.float64)
    assert int(cache.status.item()) == 0 and not cache.split_done.any()
    assert np.isfinite(out).all(), (n, T, key)
    _, cached, oc = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0] if n else 0, bits, sliding, Wk[0])
    values = np.concatenate([cached, v_new[0, 0].astype(np.float64)])
    norms = np.linalg.norm(values, axis=1)
    s0 = -256.0 * key / np.sqrt(128.0)
    S, P = (oc["S"], oc["P"]) if P0 is None else (np.zeros((256, 128)), np.full(256, P0))
    for h in range(H_q):
        phi = o_cache.feature_map(q[0, h].astype(np.float64), Wq[h].astype(np.float64))[0]
        c_n, c_d = phi @ S @ hadamard.orthonormal(128).T, phi @ P
        a, b = (np.exp(s0), 1.0) if c_d != 0 else (1.0, 0.0)
        for i in range(T):
            seen = n + i + 1
            den = a * seen + b * c_d
            y = (a * values[:seen].sum(0) + b * c_n) / den
            spread, added = a * norms[:seen].sum() / den, b * (phi @ np.linalg.norm(S, axis=1)) / den
            # roundings to binary16, half a step each: the output; weights and values; features and states, and the features as weights of the
            # divisor.  The exponent, some log2(e) |s0| large, is rounded four times to 2^-24 of it: the parts' weight against each other.
            tol = 3 * ref.HALF_STEP * np.linalg.norm(y) + 2 * ref.HALF_STEP * (spread + added) + 1.45 * abs(s0) * 2.0 ** -22 * (spread + added)
            tol += 128 ** 0.5 * 2.0 ** -25  # (a subnormal output)
            assert np.linalg.norm(out[0, h, i] - y) <= tol, (n, T, key, h, i, np.linalg.norm(out[0, h, i] - y), tol)


@pytest.mark.parametrize("bits, sliding", [(2, False), (4, False), (2, True)])
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("n, bound", [(0, 0), (0, 1), (100, 0), (100, 128), (300, 0), (300, 300), (3000, 0)])
def test_logits_far_below_zero(n, bound, T, bits, sliding):
    for key in KEYS:
        run(n, T, bits, key, sliding=sliding, bound=bound)


# P = P0 in every feature: C_d = 2 P0 (each half of phi sums to 1), S = 0: C_n = 0.
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("n, bits", [(100, 2), (300, 2), (300, 4), (3000, 2)])
@pytest.mark.parametrize("P0", [2.0 ** -20, 2.0 ** -100, 2.0 ** -130])
def test_a_correction_as_small_as_the_sum(n, bits, T, P0):
    for key in KEYS[:-1]:
        run(n, T, bits, key, P0=P0)
