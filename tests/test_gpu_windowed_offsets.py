"""Windowed decode of keys with a large offset in some channels (a bias of the key projection): a part of every score that the softmax does not see."""
import numpy as np
import pytest

from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H_q, bits", [(4, 2), (4, 4), (7, 2), (8, 4)])
@pytest.mark.parametrize("offset", [0, 30, 300, 2000])
@pytest.mark.parametrize("window, sinks", [(0, 0), (900, 130)])
def test_offsets_of_keys(H_q, bits, offset, window, sinks):
    n = 1700
    K, V, q, _, _ = ref.inputs(1030, 1, H_q, 1, [n], 1)
    e = np.zeros(128)
    e[[5, 40, 77, 120]] = offset * np.array([1.0, -1.0, 0.5, 1.0])
    K = [[(K[0][0].astype(np.float64) + e).astype(np.float16)]]
    cache = filled(1, H_q, 1, K, V, 2048, bits)
    assert cache.status.item() == 0
    got = cache.decode_windowed(to_dev(q[:, :, 0]), window, sinks=sinks).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0], bits)
    for h in range(H_q):
        # the same softmax without the offsets, and binary32's share of them in the scores: sums of 128 terms and the exponents, 2^-20 together
        y, tol = ref.attend(q[0, h], keys - e, values, [n - 1], window, sinks)
        d = 2.0 ** -20 * (np.abs(q[0, h].astype(np.float64)) @ np.abs(e))[0] / np.sqrt(128.0)
        err = np.linalg.norm(got[0, h] - y[0])
        assert err <= tol[0] + 2 * d * np.linalg.norm(values, axis=1).max(), (h, err, tol)
        # independent roundings of 2^-12 each come to far less than the bound
        assert err <= 2e-3 * np.linalg.norm(y[0]), (h, err / np.linalg.norm(y[0]))
