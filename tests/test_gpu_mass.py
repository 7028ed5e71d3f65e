"""Accumulated attention weight against the 64-bit reference: of a decode step, with its output, and of many rows; lengths, head layouts, widths, static
caches with a partial group, sliding values, ragged rows, magnitudes, bounds."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import bounded_reference as bounded
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_context_use import replayed
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu


def prepared(config, H_q, H_kv, lengths, T, bits=2, sliding=False, keep=0, R=128, scale=1.0, key_scale=1.0, room=0):
    """(cache, K, V, queries [B, H_q, T, 128], quantized tokens of each sequence)."""
    B = len(lengths)
    K, V, q, _, _ = ref.inputs(config, B, H_q, H_kv, lengths, T, scale)
    if key_scale != 1.0:
        K = [[(k.astype(np.float32) * key_scale).astype(np.float16) for k in heads] for heads in K]
    cache = filled(B, H_q, H_kv, K, V, room or max(lengths) + 128, bits, kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0, keep=keep, R=R)
    nq = [(max(n - keep, 0) if keep else o_cache.window_split(n)[0]) if n else 0 for n in lengths]
    return cache, K, V, q, nq


def prior_of(cache, seed=1):
    gen = torch.Generator().manual_seed(seed)
    return torch.rand(cache.B, cache.H_kv, cache.max_groups + 1, generator=gen).cuda()


def check_all(cache, K, V, q, nq, rows, got, prior, decay, bits, terms=1.0):
    """Masses of all pairs.  q [B, H_q, T, 128], the first rows[b] of them; they are the newest tokens."""
    gq = cache.H_q // cache.H_kv
    got = got.cpu().numpy()
    before = np.zeros_like(got) if prior is None else prior.cpu().numpy().astype(np.float64)
    num = den = 0.0
    for b in range(cache.B):
        n, r = len(K[b][0]), rows[b]
        for g in range(cache.H_kv):
            keys, _, oc = ref.tokens_of(K[b][g], V[b][g], nq[b], bits)
            slots, count, size = (np.zeros(0, int), 1, np.zeros((0, 128))) if n == 0 else bounded.slots_of(oc)
            fresh, off = np.zeros(count), np.zeros(count)
            if n and r:
                x = q[b, g * gq:(g + 1) * gq, :r].reshape(-1, 128)
                fresh, off = bounded.weights(x, keys, np.tile(n - r + np.arange(r), gq), slots, count, size)
                assert abs(fresh.sum() - gq * min(r, n)) < 1e-6
            a, w = bounded.check_mass(got[b, g, :count], before[b, g, :count], decay, fresh, off, (b, g))
            num, den = num + a, den + w
            assert (got[b, g, count:] == 7.0).all()  # not touched
    # the roundings have no common direction: 256 of 2^-24 of up to some 30 (a score's terms, `terms` times as large), which leave about 16 * 2^-24 * 30,
    # 3e-5 at most in a weight
    assert den == 0 or (num / den) ** 0.5 <= 3e-5 * max(1.0, terms), (num / den) ** 0.5


def run_rows(config, H_q, H_kv, lengths, rows, bits=2, decay=1.0, prior=True, bound=0, **over):
    T = max(max(rows), 1)
    cache, K, V, q, nq = prepared(config, H_q, H_kv, lengths, T, bits, **over)
    for b, r in enumerate(rows):
        q[b, :, r:] = np.nan  # not read
    mass = prior_of(cache) if prior else None
    out = torch.full((cache.B, H_kv, cache.max_groups + 1), 7.0, device="cuda")
    n_rows = None if all(r == T for r in rows) else to_dev(np.asarray(rows, np.int32))
    got = cache.attention_mass(to_dev(q), mass, n_rows=n_rows, decay=decay, mass_out=out, max_context=bound)
    assert got is out and cache.status.item() == 0
    check_all(cache, K, V, q, nq, rows, got, mass if decay else None, decay, bits, over.get("scale", 1.0) * over.get("key_scale", 1.0))


def run_decode(config, H_q, H_kv, lengths, bits=2, decay=1.0, prior=True, bound=0, sliding=False, check_out=True, **over):
    cache, K, V, q, nq = prepared(config, H_q, H_kv, lengths, 1, bits, sliding, **over)
    gq = H_q // H_kv
    mass = prior_of(cache) if prior else None
    out = torch.full((cache.B, H_q, 128), 7.0, dtype=torch.float16, device="cuda")
    mass_out = torch.full((cache.B, H_kv, cache.max_groups + 1), 7.0, device="cuda")
    got = cache.decode_mass(to_dev(q[:, :, 0]), mass, decay=decay, mass_out=mass_out, out=out, max_context=bound)
    assert got is out and cache.status.item() == 0 and int(cache.split_done.abs().sum()) == 0
    check_all(cache, K, V, q, nq, [1] * cache.B, mass_out, mass if decay else None, decay, bits, over.get("scale", 1.0) * over.get("key_scale", 1.0))
    got = got.cpu().numpy()
    num = den = 0.0
    for b, n in enumerate(lengths):
        if n == 0:
            assert (got[b] == 0).all()
            continue
        for g in range(H_kv if check_out else 0):
            keys, values, _ = ref.tokens_of(K[b][g], V[b][g], nq[b], bits, sliding)
            for h in range(g * gq, (g + 1) * gq):
                y, tol = ref.attend(q[b, h], keys, values, [n - 1])
                d2, y2 = ref.check_rows(got[b, h][None], y, tol, (config, b, h))
                num, den = num + d2, den + y2
    assert den == 0 or (num / den) ** 0.5 <= 2e-3


# ---- of a decode step --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("n", [1, 2, 33, 127, 128, 129, 256, 257, 300, 1000, 2500])
def test_decode_lengths(n, bits):
    run_decode(1100 + n, 8, 2, [n], bits)


@pytest.mark.parametrize("H_q, H_kv", [(1, 1), (2, 1), (3, 1), (4, 4), (8, 2), (5, 1), (6, 1), (12, 2), (7, 1), (16, 2), (3, 3)])
@pytest.mark.parametrize("bits", [2, 4])
def test_decode_head_layouts(H_q, H_kv, bits):
    run_decode(1200 + H_q, H_q, H_kv, [500, 131, 0, 64], bits, decay=0.5)


@pytest.mark.parametrize("lengths, H_q, H_kv", [([6000, 40, 900, 0, 2300], 4, 1), ([130, 8300, 131], 10, 2), ([5000] * 7 + [4871], 3, 3), ([0, 0, 1500, 0], 2, 2),
                                                ([600 - 7 * i for i in range(64)], 2, 1), ([(37 * i) % 800 for i in range(70)], 1, 1)])
def test_decode_of_uneven_batches(lengths, H_q, H_kv):
    for bound in (0, max(lengths), 500):
        run_decode(1230 + len(lengths), H_q, H_kv, lengths, 2, decay=0.5, bound=bound)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("bound", [0, 1, 700, 1 << 30])
def test_decode_bounds_size_the_launch_only(bound, bits):
    run_decode(1300, 8, 2, [700, 129, 300, 0], bits, bound=bound)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("gq", [2, 6])
def test_decode_sliding_values(bits, gq):
    run_decode(1310, 2 * gq, 2, [300, 256, 130, 90, 385, 1], bits, sliding=True)


@pytest.mark.parametrize("keep, R, n", [(1, 128, 300), (32, 32, 100), (60, 64, 513), (4, 4, 3), (128, 128, 640)])
def test_decode_static_caches_with_a_partial_group(keep, R, n):
    run_decode(1320, 8, 2, [n, n - 3 if n > 3 else n], keep=keep, R=R)


def test_decode_of_many_pairs_and_splits():
    run_decode(1330, 4, 2, [int(n) for n in np.random.default_rng(4).integers(0, 700, size=70)])  # more than 64 sequences
    run_decode(1331, 2, 1, [20000])                                                                # 32 splits


@pytest.mark.parametrize("decay, prior", [(0.0, True), (0.0, False), (1.0, False), (0.25, True)])
def test_decay_and_no_mass_before(decay, prior):
    run_decode(1340, 8, 2, [400, 1], decay=decay, prior=prior)
    run_rows(1340, 8, 2, [400, 3], [5, 5], decay=decay, prior=prior)


def test_a_decay_of_zero_does_not_read():
    cache, _, _, q, _ = prepared(1341, 8, 2, [300, 0], 1)
    bad = torch.full_like(cache.new_mass(), float("nan"))
    cache.decode_mass(to_dev(q[:, :, 0]), bad, decay=0.0)
    assert torch.isfinite(bad[0, :, :3]).all() and (bad[1, :, 0] == 0).all() and bad[0, :, 3:].isnan().all()
    bad.fill_(float("nan"))
    cache.attention_mass(to_dev(q), bad, decay=0.0)
    assert torch.isfinite(bad[0, :, :3]).all() and (bad[1, :, 0] == 0).all() and bad[1, :, 1:].isnan().all()


# Scores of hundreds, and of thousands, where single tokens have all the weight; all of them far below zero; keys and queries of extreme magnitudes
@pytest.mark.parametrize("scale, key_scale", [(20.0, 1.0), (400.0, 8.0), (1e-3, 1.0), (2.0 ** -14, 64.0), (1.0, 1200.0), (500.0, 1500.0), (0.05, 2.0 ** -12)])
@pytest.mark.parametrize("bits", [2, 4])
def test_magnitudes(scale, key_scale, bits):
    run_decode(1350, 8, 2, [700, 200], bits, scale=scale, key_scale=key_scale, check_out=False)
    run_rows(1351, 8, 2, [700, 200], [20, 7], bits, scale=scale, key_scale=key_scale)


def test_logits_far_below_zero():
    # every key the same large multiple of the negative query but for small differences: logits around -5000
    rng = np.random.default_rng(11)
    q = (np.sign(rng.standard_normal((1, 4, 1, 128))) * 20).astype(np.float16)
    K = [[(-22.0 * np.sign(q[0, 0, 0]) + rng.standard_normal((400, 128)) * 0.1).astype(np.float16) for _ in range(1)]]
    V = [[rng.standard_normal((400, 128)).astype(np.float16)]]
    cache = filled(1, 4, 1, K, V, 512)
    nq = [o_cache.window_split(400)[0]]
    got = torch.full_like(cache.new_mass(), 7.0)
    cache.decode_mass(to_dev(q[:, :, 0]), None, mass_out=got)
    check_all(cache, K, V, q, nq, [1], got, None, 1.0, 2, terms=440.0)
    got.fill_(7.0)
    cache.attention_mass(to_dev(q), None, mass_out=got)
    check_all(cache, K, V, q, nq, [1], got, None, 1.0, 2, terms=440.0)


def test_a_query_that_is_not_finite_stays_in_its_pair():
    cache, _, _, q, _ = prepared(1360, 8, 2, [300, 700, 40], 3)
    want = cache.attention_mass(to_dev(q))
    good = cache.new_mass()
    out = cache.decode_mass(to_dev(q[:, :, 0]), good)
    bad = q.copy()
    bad[1, 2, 0, 5], bad[2, 7, 0, 100] = np.nan, np.nan
    m = cache.attention_mass(to_dev(bad))
    n = cache.new_mass()
    o = cache.decode_mass(to_dev(bad[:, :, 0]), n)
    for got, ok in ((m, want), (n, good)):
        assert got[1, 0, :6].isnan().all() and got[2, 1, 0].isnan()
        same = torch.ones(3, 2, dtype=torch.bool)
        same[1, 0] = same[2, 1] = False
        assert torch.equal(got[same.cuda()], ok[same.cuda()])
    assert o[1, 2].isnan().all() and o[2, 7].isnan().all()
    keep = torch.ones(3, 8, dtype=torch.bool)
    keep[1, :4] = keep[2, 4:] = False
    assert torch.equal(o[keep.cuda()], out[keep.cuda()])
    for b, h in ((1, 0), (1, 1), (1, 3), (2, 4), (2, 5), (2, 6)):  # (the other heads of these pairs, whose query may be taken another way)
        torch.testing.assert_close(o[b, h], out[b, h], rtol=2.0 ** -9, atol=2e-3)


# ---- of many rows ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("n, T", [(1, 1), (1, 4), (5, 5), (128, 1), (129, 3), (129, 129), (300, 17), (300, 300), (257, 400), (1000, 33), (1500, 150)])
def test_rows_lengths(n, T, bits):
    run_rows(1400 + n, 8, 2, [n], [T], bits)


@pytest.mark.parametrize("H_q, H_kv", [(1, 1), (2, 1), (3, 1), (4, 4), (12, 2), (5, 1), (7, 1), (16, 2)])
@pytest.mark.parametrize("T", [1, 6, 50])
def test_rows_head_layouts(H_q, H_kv, T):
    run_rows(1500 + H_q, H_q, H_kv, [500, 131, 10], [T, max(1, T - 3), T])


@pytest.mark.parametrize("bits", [2, 4])
def test_ragged_rows(bits):
    run_rows(1510, 8, 2, [700, 0, 300, 129, 40, 1, 1000], [30, 0, 1, 64, 64, 5, 0], bits, decay=0.75)


@pytest.mark.parametrize("keep, R, n", [(1, 128, 300), (32, 32, 100), (60, 64, 513), (128, 128, 640)])
@pytest.mark.parametrize("T", [1, 40, 150])
def test_rows_over_static_caches(keep, R, n, T):
    run_rows(1520, 8, 2, [n, n - 3], [T, T], keep=keep, R=R)


def test_rows_sliding_values():
    run_rows(1530, 8, 2, [300, 90], [7, 100], sliding=True)


@pytest.mark.parametrize("H_q, H_kv, lengths, T", [(8, 1, [9000], 64), (4, 2, [3000, 2000, 10, 600], 300), (2, 1, [700] * 40, 9)])
def test_rows_of_larger_calls(H_q, H_kv, lengths, T):
    run_rows(1540, H_q, H_kv, lengths, [min(T, n) for n in lengths])


@pytest.mark.parametrize("lengths, T, bits", [([4000], 20, 2), ([3000, 4100, 77], 13, 4), ([1500 - 40 * i for i in range(33)] + [0], 20, 2), ([2500, 2300], 200, 2)])
def test_rows_where_their_sums_fit_and_where_not(lengths, T, bits):
    run_rows(1590 + T, 8, 1, lengths, [min(T, n) if i % 5 != 3 else 0 for i, n in enumerate(lengths)], bits, bound=max(lengths))


def test_a_bound_that_is_true():
    for bound in (700, 701, 900):
        run_rows(1550, 8, 2, [700, 300], [9, 9], bound=bound, room=4096)


def test_a_sequence_beyond_the_bound_adds_nothing():
    cache, K, V, q, nq = prepared(1551, 8, 2, [700, 300, 128], 4)
    mass = prior_of(cache)
    want = cache.attention_mass(to_dev(q), mass, decay=0.5, mass_out=torch.zeros_like(mass))
    got = cache.attention_mass(to_dev(q), mass, decay=0.5, mass_out=torch.zeros_like(mass), max_context=300)
    assert cache.status.item() == kv.KVLINC_ST_BOUND
    assert torch.equal(got[0, :, :6], 0.5 * mass[0, :, :6]) and (got[0, :, 6:] == 0).all()
    torch.testing.assert_close(got[1:], want[1:], rtol=1e-5, atol=0)


def test_counts_of_rows_beyond_their_range():
    cache, _, _, q, _ = prepared(1552, 8, 2, [300, 300], 4)
    mass = prior_of(cache)
    n = torch.tensor([-3, 400], dtype=torch.int32, device="cuda")
    got = cache.attention_mass(to_dev(q), mass, n_rows=n, mass_out=torch.zeros_like(mass))
    assert torch.equal(got[0, :, :3], mass[0, :, :3])
    assert torch.equal(got[1], cache.attention_mass(to_dev(q), mass, mass_out=torch.zeros_like(mass))[1])


def test_a_row_alone_and_a_decode_step_agree():
    cache, K, V, q, nq = prepared(1560, 12, 2, [1500, 129, 77], 1)
    a, b = cache.new_mass(), cache.attention_mass(to_dev(q))
    cache.decode_mass(to_dev(q[:, :, 0]), a)
    torch.testing.assert_close(a, b, rtol=3e-5, atol=1e-9)
    torch.testing.assert_close(b.sum(-1), torch.full((3, 2), 6.0, device="cuda"), rtol=1e-5, atol=0)


# ---- as a program calls them ---------------------------------------------------------------------------------------------------------

def test_in_place_twice():
    cache, K, V, q, nq = prepared(1570, 8, 2, [700, 5], 3)
    mass = prior_of(cache)
    once = cache.attention_mass(to_dev(q), mass, decay=0.5, mass_out=torch.zeros_like(mass))
    twice = cache.attention_mass(to_dev(q), once, decay=0.5, mass_out=torch.zeros_like(mass))
    assert cache.attention_mass(to_dev(q), mass, decay=0.5) is mass
    cache.attention_mass(to_dev(q), mass, decay=0.5)
    assert torch.equal(mass[0, :, :6], twice[0, :, :6]) and torch.equal(mass[1, :, :1], twice[1, :, :1])
    q1 = to_dev(q[:, :, 0])
    mass, other = prior_of(cache), prior_of(cache)
    a = cache.decode_mass(q1, mass, decay=0.5)
    b = cache.decode_mass(q1, other, decay=0.5, mass_out=other, out=q1)
    assert b is q1 and torch.equal(a, b) and torch.equal(mass, other)


def test_the_same_bits_in_every_run():
    cache, _, _, q, _ = prepared(1580, 8, 2, [5000, 300, 4000], 40)
    first = None
    for _ in range(4):
        m = cache.attention_mass(to_dev(q))
        n = cache.new_mass()
        o = cache.decode_mass(to_dev(q[:, :, 0]), n)
        first = first or (m, n, o)
        assert all(torch.equal(a, b) for a, b in zip(first, (m, n, o)))


def test_from_a_graph():
    cache, _, _, _, _ = prepared(1590, 8, 2, [3000, 127], 1, room=4096)
    q, q1 = torch.zeros(2, 8, 20, 128, dtype=torch.float16, device="cuda"), torch.zeros(2, 8, 128, dtype=torch.float16, device="cuda")
    row = torch.zeros(2, 2, 1, 128, dtype=torch.float16, device="cuda")
    prior = prior_of(cache)
    bufs = [[torch.zeros_like(prior), torch.zeros_like(prior), torch.zeros_like(q1)] for _ in range(2)]

    def call(b):
        for t in b:  # (slots beyond the window's stay as they are)
            t.zero_()
        cache.attention_mass(q, prior, decay=0.5, mass_out=b[0])
        cache.decode_mass(q1, prior, mass_out=b[1], out=b[2])
        return b

    def prepare(i):
        for t in (q, q1, row):
            t.normal_()
        cache.append(row, row)
        prior.uniform_()

    def eager():
        call(bufs[1])
        return [t.view(torch.int16) for t in bufs[1]]

    replayed(lambda: [t.view(torch.int16) for t in call(bufs[0])], prepare, eager)


def test_two_caches_on_two_streams():
    made = [prepared(1600 + i, 8, 2, [2000 + 500 * i, 300], 16) for i in range(2)]
    q = [to_dev(m[3]) for m in made]
    want = [(m[0].attention_mass(x), m[0].new_mass(), ) for m, x in zip(made, q)]
    outs = [m[0].decode_mass(x[:, :, 0].contiguous(), w[1]) for m, x, w in zip(made, q, want)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for turn in range(5):
        for m, x, s in zip(made, q, streams):
            mass = m[0].attention_mass(x, stream=s)
            with torch.cuda.stream(s):
                one, q1 = m[0].new_mass(), x[:, :, 0].contiguous()
            got.append((mass, one, m[0].decode_mass(q1, one, stream=s)))
    torch.cuda.synchronize()
    for i, (mass, one, out) in enumerate(got):
        assert torch.equal(mass, want[i % 2][0]) and torch.equal(one, want[i % 2][1]) and torch.equal(out, outs[i % 2])
