"""Few-row prompt attention: the largest scale of a group in every place that a record has for it, of keys (per channel) and of values (per token)."""
import numpy as np
import pytest
import torch

import kvlinc_synth as synth
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def run_case(K, V, q, bits):
    """One pair of one KV head and 4 query heads: rows q [4, T, 128] over 200 cached tokens and T new rows."""
    T = q.shape[1]
    cache = filled(1, 4, 1, [[K[:200]]], [[V[:200]]], 512, bits)
    k_new, v_new = K[None, None, 200:200 + T], V[None, None, 200:200 + T]
    got = cache.prompt_attention(to_dev(q[None]), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[:200], V[:200], 128, bits)
    keys = np.concatenate([keys, k_new[0, 0].astype(np.float64)])
    values = np.concatenate([values, v_new[0, 0].astype(np.float64)])
    for h in range(4):
        y, tol = ref.attend(q[h], keys, values, 200 + np.arange(T))
        ref.check_rows(got[0, h], y, tol, (bits, h))


def inputs(config, T):
    q = np.stack([synth.queries(config, 0, 4, step=i) for i in range(T)], 1)
    return synth.keys(config, 0, 0, 210), synth.values(config, 0, 0, 210), q


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [1, 2, 6])
@pytest.mark.parametrize("channel", [0, 1, 2, 3, 4, 5, 6, 7, 70, 71, 123, 126])
def test_a_channel_of_large_keys(channel, T, bits):
    # the query's largest number on the channel whose scale is 2^11 or more: their product leaves binary16's range at the query's usual scale
    K, V, q = inputs(1010, T)
    K = K.astype(np.float32) * 0.5
    K[:, channel] = np.random.default_rng(channel).choice([-1.0, 1.0], 210) * 20000.0
    q = q.astype(np.float32) * 2.0 ** -12
    q[:, :, channel] = 1.9 * 2.0 ** -12
    run_case(K.astype(np.float16), V, q.astype(np.float16), bits)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [1, 2, 6])
@pytest.mark.parametrize("token", [0, 15, 16, 17, 35, 50, 64, 81, 99, 127])
def test_a_token_of_large_values(token, T, bits):
    K, V, q = inputs(1020, T)
    V = V.astype(np.float32) * 2.0 ** -10
    V[token] *= 2.0 ** 21
    K = K.astype(np.float32) * 0.1
    # (the row that sees it most: its weight is near the largest)
    K[token] = q[0, 0].astype(np.float32) * 0.3
    run_case(K.astype(np.float16), V.astype(np.float16), q, bits)
