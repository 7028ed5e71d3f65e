"""Windowed decode against the 64-bit reference, and against the decode over everything."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def run_case(config, H_q, H_kv, lengths, window, sinks, bits=2, sliding=False, keep=0, R=128, bound=0):
    B, gq = len(lengths), H_q // H_kv
    K, V, q, _, _ = ref.inputs(config, B, H_q, H_kv, lengths, 1)
    cache = filled(B, H_q, H_kv, K, V, max(lengths) + 128, bits, kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0, keep=keep, R=R)
    q = q[:, :, 0]
    out = torch.full((B, H_q, 128), 7.0, dtype=torch.float16, device="cuda")
    got = cache.decode_windowed(to_dev(q), window, sinks=sinks, out=out, max_context=bound)
    assert got is out and int(cache.split_done.abs().sum()) == 0
    got = got.cpu().numpy()
    num = den = 0.0
    for b in range(B):
        n = lengths[b]
        if n == 0:
            assert (got[b] == 0).all()
            continue
        nq = max(n - keep, 0) if keep else o_cache.window_split(n)[0]
        for g in range(H_kv):
            keys, values, _ = ref.tokens_of(K[b][g], V[b][g], nq, bits, sliding)
            for h in range(g * gq, (g + 1) * gq):
                y, tol = ref.attend(q[b, h][None], keys, values, [n - 1], window, sinks)
                d2, y2 = ref.check_rows(got[b, h][None], y, tol, (config, b, h))
                num, den = num + d2, den + y2
    assert den == 0 or (num / den) ** 0.5 <= 2e-3


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 0), (1, 1), (2, 0), (17, 4), (128, 0), (129, 1), (250, 130), (400, 3), (3000, 0), (60, 2000)])
def test_windows_and_sinks(window, sinks, bits):
    run_case(900, 8, 2, [700, 1, 128, 129, 0, 300], window, sinks, bits)


@pytest.mark.parametrize("H_q, H_kv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (12, 2), (7, 1), (16, 2), (4, 4)])
def test_head_layouts(H_q, H_kv):
    run_case(910, H_q, H_kv, [500, 131], 200, 4)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("window", [0, 1, 60, 128, 140, 300])
def test_sliding_values(window, bits):
    run_case(920, 8, 2, [300, 256, 130, 90, 385], window, 3, bits, sliding=True)


@pytest.mark.parametrize("keep, R, n", [(1, 128, 300), (32, 32, 100), (60, 64, 513)])
@pytest.mark.parametrize("window, sinks", [(0, 0), (20, 5), (90, 0)])
def test_static_caches_with_a_partial_group(keep, R, n, window, sinks):
    run_case(930, 8, 2, [n, n - 3], window, sinks, keep=keep, R=R)


@pytest.mark.parametrize("lengths", [[5000], [6000, 2300, 40], [4097] * 3])
@pytest.mark.parametrize("window", [0, 2500])
def test_long_contexts_in_splits(lengths, window):
    run_case(940, 8, 2, lengths, window, 130)


@pytest.mark.parametrize("bits", [2, 4])
def test_without_a_limit_it_is_the_decode_over_everything(bits):
    B, H_q, H_kv, lengths = 3, 8, 2, [1500, 300, 129]
    K, V, q, _, _ = ref.inputs(950, B, H_q, H_kv, lengths, 1)
    cache = filled(B, H_q, H_kv, K, V, 2048, bits)
    q = to_dev(q[:, :, 0])
    want = cache.decode(q).float()
    for window, sinks in ((0, 0), (1500, 0), (1 << 30, 7), (2 ** 31 - 1, 2 ** 31 - 1)):
        got = cache.decode_windowed(q, window, sinks=sinks).float()
        assert ((got - want).norm() / want.norm()).item() < 2e-3


def test_the_same_call_gives_the_same_bits():
    B, H_q, H_kv, lengths = 2, 8, 2, [3000, 700]
    K, V, q, _, _ = ref.inputs(960, B, H_q, H_kv, lengths, 1)
    cache = filled(B, H_q, H_kv, K, V, 4096)
    q = to_dev(q[:, :, 0])
    a = cache.decode_windowed(q, 2000, sinks=4)
    for _ in range(5):
        assert torch.equal(cache.decode_windowed(q, 2000, sinks=4), a)
