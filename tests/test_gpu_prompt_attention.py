"""Prompt attention against the 64-bit reference: lengths from one token on, ragged rows, windows and sinks, both widths, every head layout,
static caches with a partial group, the correction, and rows behind the last one."""
import numpy as np
import pytest
import torch

import kvlinc_synth as synth
import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev

pytestmark = pytest.mark.gpu


def filled(B, H_q, H_kv, K, V, room, bits=2, flags=0, Wq=None, Wk=None, keep=0, R=128):
    lengths = [len(K[b][0]) for b in range(B)]
    cache = kv.KVLincCache(B, H_q, H_kv, room, R=R, Wq=Wq, Wk=Wk, bits=bits, flags=flags)
    if max(lengths):
        T = max(lengths)
        pad = np.zeros((B, H_kv, T, 128), np.float16)
        pad_v = pad.copy()
        for b in range(B):
            for g in range(H_kv):
                pad[b, g, :lengths[b]], pad_v[b, g, :lengths[b]] = K[b][g], V[b][g]
        cache.append(to_dev(pad), to_dev(pad_v), n_new=to_dev(np.asarray(lengths, np.int32)), keep_residual=keep)
        assert cache.status.item() == 0
    return cache


def run_case(config, H_q, H_kv, lengths, rows, bits=2, window=0, sinks=0, corr=False, sliding=False, keep=0, R=128, scale=1.0, bound=0):
    B, T, gq = len(lengths), max(max(rows), 1), H_q // H_kv
    K, V, q, k_new, v_new = ref.inputs(config, B, H_q, H_kv, lengths, T, scale)
    Wq, Wk = (synth.adapters_q(config, H_q), synth.adapters_k(config, H_kv)) if corr else (None, None)
    cache = filled(B, H_q, H_kv, K, V, max(lengths) + 128, bits, kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0,
                   None if Wq is None else to_dev(Wq), None if Wk is None else to_dev(Wk), keep, R)
    # rows behind the last one of a sequence: not a number, and an output that has to stay
    for b in range(B):
        q[b, :, rows[b]:] = np.nan
        k_new[b, :, rows[b]:] = np.inf
        v_new[b, :, rows[b]:] = np.nan
    out = torch.full((B, H_q, T, 128), 7.0, dtype=torch.float16, device="cuda")
    ragged = any(r != T for r in rows)
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new), n_new=to_dev(np.asarray(rows, np.int32)) if ragged else None,
                                 window=window, sinks=sinks, out=out, max_context=bound)
    assert got is out and int(cache.split_done.abs().sum()) == 0
    got = got.cpu().numpy()
    num = den = 0.0
    for b in range(B):
        n, r = lengths[b], rows[b]
        assert (got[b, :, r:] == 7.0).all()
        nq = (max(n - keep, 0) if keep else o_cache.window_split(n)[0]) if n else 0
        for g in range(H_kv):
            keys, values, oc = ref.tokens_of(K[b][g], V[b][g], nq, bits, sliding, Wk[g] if corr else None)
            keys = np.concatenate([keys, k_new[b, g, :r].astype(np.float64)])
            values = np.concatenate([values, v_new[b, g, :r].astype(np.float64)])
            for h in range(g * gq, (g + 1) * gq):
                if r == 0:
                    continue
                y, tol = ref.attend(q[b, h, :r], keys, values, n + np.arange(r), window, sinks, oc, Wq[h] if corr else None)
                d2, y2 = ref.check_rows(got[b, h, :r], y, tol, (config, b, h))
                num, den = num + d2, den + y2
    assert den == 0 or (num / den) ** 0.5 <= 2e-3, (num / den) ** 0.5


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("n, T", [(0, 1), (0, 2), (0, 31), (0, 130), (1, 1), (5, 3), (128, 4), (129, 5), (300, 1), (300, 33), (257, 70), (1000, 6)])
def test_lengths(n, T, bits):
    run_case(700 + n, 8, 2, [n], [T], bits)


@pytest.mark.parametrize("H_q, H_kv", [(1, 1), (2, 1), (6, 2), (4, 1), (5, 1), (12, 2), (7, 1), (8, 1), (3, 3)])
@pytest.mark.parametrize("T", [1, 4, 40])
def test_head_layouts(H_q, H_kv, T):
    run_case(800 + H_q, H_q, H_kv, [260, 131], [T, max(1, T - 3)])


@pytest.mark.parametrize("bits", [2, 4])
def test_ragged_batch(bits):
    run_case(810, 8, 2, [0, 700, 129, 1, 256, 128], [9, 0, 17, 1, 5, 16], bits)


def test_ragged_batch_of_many_rows():
    run_case(811, 4, 1, [0, 300, 0, 129], [200, 77, 0, 150])


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (2, 3), (16, 0), (100, 5), (128, 128), (129, 130), (200, 1000), (5000, 4), (300, 0)])
@pytest.mark.parametrize("T", [1, 5, 60])
def test_windows(window, sinks, T):
    run_case(820, 8, 2, [900, 40, 0], [T, T, max(1, T // 2)], 2, window, sinks)


@pytest.mark.parametrize("window, sinks", [(3, 1), (150, 260)])
def test_windows_of_four_bits(window, sinks):
    run_case(821, 4, 2, [700, 129], [20, 7], 4, window, sinks)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("H_q, H_kv, T", [(8, 2, 1), (8, 2, 5), (7, 1, 40), (2, 2, 33), (4, 4, 16)])
def test_correction(H_q, H_kv, T, bits):
    run_case(830, H_q, H_kv, [700, 100, 0, 257], [T, T, T, max(1, T - 2)], bits, corr=True)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("window", [0, 90, 200])
def test_sliding_values(bits, window):
    run_case(840, 8, 2, [300, 256, 130, 90], [6, 40, 3, 5], bits, window, 2 if window else 0, sliding=True)


@pytest.mark.parametrize("keep, R, n", [(1, 128, 300), (32, 32, 100), (128, 128, 200), (60, 64, 513), (4, 4, 130)])
@pytest.mark.parametrize("window", [0, 50])
def test_static_caches_with_a_partial_group(keep, R, n, window):
    run_case(850, 8, 2, [n, n - 3], [5, 20], 2, window, 3, keep=keep, R=R)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("n, T", [(0, 129), (0, 300), (1, 130), (128, 200), (300, 129), (1000, 260)])
def test_more_rows_than_a_few_blocks(n, T, bits):
    run_case(855, 8, 1, [n], [T], bits)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (30, 3), (64, 64), (100, 5), (129, 130), (200, 1000), (5000, 4), (700, 0)])
def test_windows_of_many_rows(window, sinks):
    run_case(856, 7, 1, [900, 40, 0, 300], [160, 170, 33, 147], 2, window, sinks)


@pytest.mark.parametrize("bits, corr, sliding", [(2, True, False), (4, True, False), (2, False, True), (4, False, True)])
def test_variants_of_many_rows(bits, corr, sliding):
    run_case(857, 8, 1, [700, 100, 0, 257], [150, 131, 129, 4], bits, corr=corr, sliding=sliding)


def test_single_heads_and_many_rows():
    run_case(858, 2, 2, [300, 129], [1100, 1030])


@pytest.mark.parametrize("keep, R, n", [(32, 32, 100), (60, 64, 513)])
def test_static_caches_and_many_rows(keep, R, n):
    run_case(859, 8, 1, [n, n - 3], [150, 140], 2, 90, 3, keep=keep, R=R)


@pytest.mark.parametrize("T", [3, 40, 300])
def test_large_and_small_scores(T):
    # scores of some hundreds and next to none: the reference of a row moves by more than its head room, or not at all
    for scale in (32.0, 2.0 ** -12, 0.0):
        run_case(860, 8, 2, [400], [T], scale=scale)


@pytest.mark.parametrize("bound", [0, 5000, 2000])
def test_the_launch_bound_changes_nothing_but_the_splits(bound):
    run_case(870, 8, 2, [2000], [4], bound=bound)


def test_scale_of_the_values():
    # value scales from subnormal to the largest: the weights carry them with the group's exponent taken out
    B, H_q, H_kv, n, T = 1, 4, 1, 300, 3
    for gain in (2.0 ** -16, 2.0 ** -8, 1000.0, 16000.0):
        K, V, q, k_new, v_new = ref.inputs(880, B, H_q, H_kv, [n], T)
        V = [[np.clip(V[0][0].astype(np.float32) * gain, -60000, 60000).astype(np.float16)]]
        v_new = np.clip(v_new.astype(np.float32) * gain, -60000, 60000).astype(np.float16)
        V[0][0] = np.clip(V[0][0], -4000, 4000) if gain > 4000 else V[0][0]  # (the rotation sums 128 of them: inside binary16)
        cache = filled(B, H_q, H_kv, K, V, 512)
        assert cache.status.item() == 0
        got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
        keys, values, _ = ref.tokens_of(K[0][0], V[0][0], 256)
        keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
        for h in range(H_q):
            y, tol = ref.attend(q[0, h], keys, values, n + np.arange(T))
            ref.check_rows(got[0, h], y, tol + 128 ** 0.5 * 2.0 ** -24, (gain, h))  # (a subnormal output: half a step of 2^-24)


def test_not_finite_rows_stay_in_their_sequence():
    B, H_q, H_kv, T = 3, 4, 1, 20
    K, V, q, k_new, v_new = ref.inputs(890, B, H_q, H_kv, [140] * B, T)
    cache = filled(B, H_q, H_kv, K, V, 512)
    want = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu()
    k_new[1, 0, 3, 5], v_new[1, 0, 7, 9] = np.inf, np.nan
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert not torch.isfinite(got[1, :, 7:]).all()
