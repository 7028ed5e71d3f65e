"""A new key or value that is not finite reaches the rows that see it, and no others: earlier rows, rows whose window has passed it."""
import numpy as np
import pytest

import kvlinc_synth as synth
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def run(config, H_q, H_kv, n, T, window=0, sinks=0, corr=False, bits=2, rows=None):
    gq, r = H_q // H_kv, T if rows is None else rows
    K, V, q, k_new, v_new = ref.inputs(config, 1, H_q, H_kv, [n], T)
    Wq, Wk = (synth.adapters_q(config, H_q), synth.adapters_k(config, H_kv)) if corr else (None, None)
    cache = filled(1, H_q, H_kv, K, V, n + 128, bits, Wq=to_dev(Wq) if corr else None, Wk=to_dev(Wk) if corr else None)
    n_new = None if rows is None else to_dev(np.asarray([rows], np.int32))
    want = []
    for g in range(H_kv):
        keys, values, oc = ref.tokens_of(K[0][g], V[0][g], o_cache.window_split(n)[0] if n else 0, bits, Wk=Wk[g] if corr else None)
        keys, values = np.concatenate([keys, k_new[0, g, :r].astype(np.float64)]), np.concatenate([values, v_new[0, g, :r].astype(np.float64)])
        want += [ref.attend(q[0, h, :r], keys, values, n + np.arange(r), window, sinks, oc, Wq[h] if corr else None) for h in range(g * gq, (g + 1) * gq)]
    i = np.arange(r)
    for g in range(H_kv):
        for j in sorted({0, 1, r // 3, r // 2, r - 2, r - 1} & set(range(r))):
            for where, bad in (("v", np.inf), ("v", -np.inf), ("v", np.nan), ("k", np.nan), ("k", np.inf), ("both", np.nan)):
                k, v = k_new.copy(), v_new.copy()
                if where != "v":
                    k[0, g, j, 17] = bad
                if where != "k":
                    v[0, g, j, 100] = bad
                got = cache.prompt_attention(to_dev(q), to_dev(k), to_dev(v), n_new=n_new, window=window, sinks=sinks).cpu().numpy()
                sees = (j <= i) & ((window == 0) | (i - j < window) | (n + j < sinks))
                for h in range(H_q):
                    y, tol = want[h]
                    clean = ~sees if h // gq == g else np.ones(r, bool)
                    ref.check_rows(got[0, h, :r][clean], y[clean], tol[clean], (g, j, where, bad, h)) if clean.any() else None
                    if where != "k" or np.isnan(bad):  # (a key with an infinite channel: a weight of 0, or not a number)
                        assert not np.isfinite(got[0, h, :r][~clean]).all(1).any(), (g, j, where, bad, h)
    assert not cache.split_done.any() and cache.status.item() == 0


@pytest.mark.parametrize("H_q, H_kv, T", [(4, 1, 3), (8, 2, 5), (1, 1, 2), (7, 1, 9), (1, 1, 64), (4, 1, 17), (4, 1, 40), (8, 1, 64), (1, 1, 300), (4, 1, 130), (8, 1, 200), (1, 1, 700)])
@pytest.mark.parametrize("n", [0, 140])
def test_rows_that_do_not_see_it_stay(H_q, H_kv, T, n):
    run(1010, H_q, H_kv, n, T)


@pytest.mark.parametrize("H_q, H_kv, T", [(4, 1, 10), (1, 1, 60), (4, 1, 100), (4, 1, 200), (1, 1, 600)])
@pytest.mark.parametrize("window, sinks", [(1, 0), (5, 142), (70, 0)])
def test_windows_that_have_passed_it(H_q, H_kv, T, window, sinks):
    run(1011, H_q, H_kv, 140, T, window, sinks)


@pytest.mark.parametrize("H_q, H_kv, T", [(8, 2, 4), (4, 1, 40), (8, 1, 70)])
@pytest.mark.parametrize("bits", [2, 4])
def test_splits_and_the_correction(H_q, H_kv, T, bits):
    run(1012, H_q, H_kv, 3000, T, corr=True, bits=bits)


@pytest.mark.parametrize("T, rows", [(12, 7), (60, 33), (300, 131), (300, 128)])
def test_the_last_rows_of_a_shorter_sequence(T, rows):
    run(1013, 4, 1, 140, T, rows=rows)
