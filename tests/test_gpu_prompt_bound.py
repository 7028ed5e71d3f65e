"""Prompt attention of sequences that hold more tokens than max_context says: right, or zeros and a bit in the status word, never part of a sum."""
import numpy as np
import pytest

import kvlinc_synth as synth
import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def check(config, lengths, rows, bound, refused, window=0, sinks=0, corr=False):
    B, H_q, H_kv, gq, T = len(lengths), 4, 1, 4, max(rows)
    K, V, q, k_new, v_new = ref.inputs(config, B, H_q, H_kv, lengths, T)
    Wq, Wk = (synth.adapters_q(config, H_q), synth.adapters_k(config, H_kv)) if corr else (None, None)
    cache = filled(B, H_q, H_kv, K, V, max(lengths) + 128, Wq=to_dev(Wq) if corr else None, Wk=to_dev(Wk) if corr else None)
    n_new = to_dev(np.asarray(rows, np.int32)) if min(rows) < T else None
    for _ in range(2):
        got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new), n_new=n_new, window=window, sinks=sinks, max_context=bound).cpu().numpy()
        assert int(cache.status.item()) == (kv.KVLINC_ST_BOUND if refused else 0) and not cache.split_done.any()
        for b in range(B):
            n, r = lengths[b], rows[b]
            assert (got[b, :, r:] == 0).all()
            if b in refused:
                assert (got[b] == 0).all()
                continue
            keys, values, oc = ref.tokens_of(K[b][0], V[b][0], o_cache.window_split(n)[0] if n else 0, Wk=Wk[0] if corr else None)
            keys = np.concatenate([keys, k_new[b, 0, :r].astype(np.float64)])
            values = np.concatenate([values, v_new[b, 0, :r].astype(np.float64)])
            for h in range(H_q):
                y, tol = ref.attend(q[b, h, :r], keys, values, n + np.arange(r), window, sinks, oc, Wq[h] if corr else None)
                ref.check_rows(got[b, h, :r], y, tol, (b, h))


@pytest.mark.parametrize("corr", [False, True])
@pytest.mark.parametrize("T", [4, 100, 128])
def test_up_to_512_rows_the_bound_only_sizes_the_launch(T, corr):
    check(1000, [700, 64, 0], [T, T, T], 64, [], corr=corr)


@pytest.mark.parametrize("corr", [False, True])
@pytest.mark.parametrize("lengths, bound, refused", [([700, 64, 0], 64, [0]), ([129, 128, 300], 128, [0, 2]), ([1, 5], 1, []), ([65, 64], 1, [0]), ([3000, 2900], 2900, [0])])
def test_more_rows_get_zeros(lengths, bound, refused, corr):
    check(1001, lengths, [129] * len(lengths), bound, refused, corr=corr)
    check(1002, lengths, [140, 131, 3][:len(lengths)], bound, refused, corr=corr)


def test_a_window_needs_no_bound():
    # the rows near the window are as many whatever a sequence holds; below them, where the bound is less than they are, it counts
    check(1003, [900, 700], [130, 129], 400, [], window=100, sinks=5)
    check(1004, [900, 30], [130, 129], 64, [0], window=100, sinks=5)
