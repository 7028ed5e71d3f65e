"""Rotary positions against the 64-bit reference: both layouts, parts of a head, every type in and out, strides, positions from counters, offsets and
depths, far ones; rows behind the last one; in place, the way back, graphs and streams."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from tests import bounded_reference as ref
from tests.test_gpu_context_use import replayed

pytestmark = pytest.mark.gpu


def inputs(B, H_q, H_kv, T, din, fused, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T, H_q + 2 * H_kv, 128, generator=gen).to(ref.TYPES[din])
    if fused:
        x = x.cuda().transpose(1, 2)
        return x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    return tuple(t.transpose(1, 2).contiguous().cuda() for t in x.split((H_q, H_kv, H_kv), 2))


def check(got, x, positions, plan, dout, turned, rows):
    """got, x [B, heads, T, 128]; positions [B, T]."""
    got, x = got.double().cpu().numpy(), x.double().cpu().numpy()
    freq = plan.freq.cpu().numpy()
    for b in range(len(x)):
        r = rows[b]
        if turned:
            y, off = ref.rotated(x[b, :, :r], positions[b][:r], freq, plan.interleaved, plan.magnitude)
        else:
            y, off = x[b, :, :r], 0.0
        d = np.abs(got[b, :, :r] - y)
        tol = off + ref.rounding(y, dout)
        assert (d <= tol).all(), (b, np.unravel_index((d - tol).argmax(), d.shape), d.max())


def run_case(B=2, H_q=8, H_kv=2, T=5, channels=128, interleaved=False, din="f16", dout="f16", fused=True, magnitude=1.0, first=None, depth=None, counted=True,
             rows=None, held=(300, 7), base=10000.0, seed=0):
    plan = kv.KVLincRotary(kv.rotary_frequencies(channels, base=base), interleaved=interleaved, magnitude=magnitude)
    cache = kv.KVLincCache(B, H_q, H_kv, 512)
    n = np.resize(np.asarray(held), B)
    cache.n_quant.copy_(torch.tensor(n // 128 * 128))
    cache.n_res.copy_(torch.tensor(n % 128))
    q, k, v = inputs(B, H_q, H_kv, T, din, fused, seed)
    real = [T] * B if rows is None else rows
    if not fused or rows is not None:  # rows behind the last one are not read
        for t in (q, k, v):
            for b in range(B):
                t[b, :, real[b]:] = float("nan")
    outs = [torch.full(t.shape, 7.0, dtype=ref.TYPES[dout], device="cuda") for t in (q, k, v)]
    ints = lambda a: None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    got = cache.rotary(plan, q, k, v, n_new=ints(rows), first=ints(first), depth=ints(depth), counted=counted, q_out=outs[0], k_out=outs[1], v_out=outs[2])
    assert all(a is b for a, b in zip(got, outs))
    at = np.zeros((B, T)) + (n[:, None] if counted else 0) + (0 if first is None else np.asarray(first, np.float64)[:, None])
    at = at + (np.arange(T) if depth is None else np.asarray(depth))
    for t, x, turned in zip(got, (q, k, v), (True, True, False)):
        check(t, x, at, plan, dout, turned, real)
        for b in range(B):
            assert (t[b, :, real[b]:] == 7.0).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("channels", [2, 4, 14, 16, 20, 32, 50, 64, 96, 112, 126, 128])
def test_parts_of_a_head(channels, interleaved):
    run_case(channels=channels, interleaved=interleaved)
    run_case(channels=channels, interleaved=interleaved, fused=False, T=1, magnitude=1.25)


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("din", list(ref.TYPES))
@pytest.mark.parametrize("dout", list(ref.TYPES))
@pytest.mark.parametrize("channels, interleaved", [(128, False), (64, True), (36, False)])
def test_types(channels, interleaved, din, dout, fused):
    run_case(channels=channels, interleaved=interleaved, din=din, dout=dout, fused=fused, T=9)


@pytest.mark.parametrize("H_q, H_kv", [(1, 1), (7, 1), (8, 1), (5, 5), (28, 4), (64, 8), (3, 3)])
@pytest.mark.parametrize("T", [1, 3, 70])
def test_head_layouts_and_lengths(H_q, H_kv, T):
    run_case(B=3, H_q=H_q, H_kv=H_kv, T=T, held=(0, 1, 300))


@pytest.mark.parametrize("B, T", [(1, 2047), (2, 1025), (300, 9)])
def test_many_tokens(B, T):
    run_case(B=B, T=T, H_q=6, H_kv=2, din="bf16", held=(0,))


@pytest.mark.parametrize("channels, interleaved", [(128, False), (96, False), (128, True), (36, False)])
@pytest.mark.parametrize("din, dout", [("f16", "f16"), ("f32", "f16"), ("bf16", "f32"), ("f32", "f32")])
def test_a_large_call_gives_what_smaller_ones_give(channels, interleaved, din, dout):
    plan, T = kv.KVLincRotary(kv.rotary_frequencies(channels), interleaved=interleaved, magnitude=0.75), 6002  # 74 MB of 2-byte results
    cache = kv.KVLincCache(1, 32, 8, 128)
    q, k, v = inputs(1, 32, 8, T, din, True)
    large = cache.rotary(plan, q, k, v, dtype=ref.TYPES[dout])
    for t0 in range(0, T, 1500):
        part = [t[:, :, t0:t0 + 1500] for t in (q, k, v)]
        small = cache.rotary(plan, *part, first=torch.tensor([t0], dtype=torch.int32, device="cuda"), dtype=ref.TYPES[dout])
        for a, b in zip(large, small):
            assert torch.equal(a[:, :, t0:t0 + 1500], b)
    if din == dout:
        mine = [t.contiguous() for t in (q, k, v)]
        cache.rotary(plan, *mine, q_out=mine[0], k_out=mine[1], v_out=mine[2])
        assert all(torch.equal(a, b) for a, b in zip(mine, large))


@pytest.mark.parametrize("interleaved, channels", [(False, 128), (True, 96), (False, 20)])
def test_ragged_rows(interleaved, channels):
    run_case(B=4, T=11, rows=[11, 0, 1, 6], interleaved=interleaved, channels=channels, held=(0, 129))


def test_counts_of_rows_beyond_their_range():
    plan = kv.KVLincRotary(kv.rotary_frequencies())
    cache = kv.KVLincCache(2, 4, 2, 128)
    q, _, _ = inputs(2, 4, 2, 6, "f16", False)
    n = torch.tensor([-5, 1000], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    cache.rotary(plan, q, n_new=n, q_out=out)
    assert (out[0] == 7.0).all() and torch.equal(out[1], cache.rotary(plan, q)[0][1])


@pytest.mark.parametrize("first, counted", [([1000000, 123456], True), ([2 ** 31 - 1, 2 ** 31 - 2], True), ([2 ** 31 - 1, 0], False), ([-5, -2 ** 31], True), ([0, 131071], False)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(first, counted, interleaved):
    run_case(first=first, counted=counted, interleaved=interleaved, din="f32", dout="f32", base=500000.0)


def test_depths_of_drafted_trees():
    run_case(B=3, T=7, depth=[[0, 1, 1, 2, 2, 2, 3], [0, 0, 0, 0, 0, 0, 0], [5, 4, 3, 2, 1, 0, -1]], first=[9, 1000, 50])
    run_case(B=2, T=3, depth=[[2 ** 31 - 1, 0, 1], [7, 7, 7]], counted=False, rows=[3, 1], dout="f32")


def test_broadcast_and_padded_strides():
    plan = kv.KVLincRotary(kv.rotary_frequencies())
    cache = kv.KVLincCache(3, 4, 2, 128)
    gen = torch.Generator().manual_seed(3)
    one = torch.randn(1, 4, 5, 128, generator=gen).half().cuda()
    wide = torch.randn(3, 2, 5, 136, generator=gen).half().cuda()[..., :128]
    q, k, _ = cache.rotary(plan, one.expand(3, -1, -1, -1), wide)
    q2, k2, _ = cache.rotary(plan, one.expand(3, -1, -1, -1).contiguous(), wide.contiguous())
    assert torch.equal(q, q2) and torch.equal(k, k2)
    with pytest.raises(kv.KVLincError):  # rows that do not begin at 16 bytes
        cache.rotary(plan, torch.zeros(3, 4, 5, 132, device="cuda").half()[..., :128])
    with pytest.raises(kv.KVLincError):
        cache.rotary(plan, torch.zeros(3 * 4 * 5 * 128 + 8, device="cuda").half()[4:-4].view(3, 4, 5, 128))


@pytest.mark.parametrize("which", ["q", "k", "v", "qk", "kv"])
def test_some_of_the_tensors(which):
    plan = kv.KVLincRotary(kv.rotary_frequencies(96))
    cache = kv.KVLincCache(2, 8, 2, 128)
    cache.n_res.fill_(5)
    all_of = dict(zip("qkv", inputs(2, 8, 2, 4, "bf16", True)))
    want = dict(zip("qkv", cache.rotary(plan, **all_of)))
    got = dict(zip("qkv", cache.rotary(plan, **{x: all_of[x] for x in which})))
    for x in "qkv":
        assert (got[x] is None) if x not in which else torch.equal(got[x], want[x])


@pytest.mark.parametrize("channels, interleaved", [(128, False), (128, True), (36, False), (64, False)])
@pytest.mark.parametrize("dtype", list(ref.TYPES))
def test_in_place_and_back(channels, interleaved, dtype):
    plan = kv.KVLincRotary(kv.rotary_frequencies(channels), interleaved=interleaved, magnitude=2.0)
    cache = kv.KVLincCache(2, 8, 2, 1024)
    cache.n_res.fill_(100)
    q, k, v = inputs(2, 8, 2, 13, dtype, False)
    want = cache.rotary(plan, q, k, v, dtype=ref.TYPES[dtype])
    x, y, z = q.clone(), k.clone(), v.clone()
    got = cache.rotary(plan, x, y, z, q_out=x, k_out=y, v_out=z)
    assert got[0] is x and all(torch.equal(a, b) for a, b in zip(got, want))
    back = cache.rotary(plan.inverse(), x, q_out=x)[0]
    # twice a rounding to the type (of numbers up to 2 sqrt(2) times as large, halved again), and the arithmetic's
    size = 2 * q.double().abs().amax()
    assert (back.double() - q.double()).abs().amax() <= 2 * torch.finfo(ref.TYPES[dtype]).eps / 2 * size + 32 * 2.0 ** -24 * size


def test_numbers_that_are_not_finite_stay_in_their_pair():
    for channels, interleaved in ((64, False), (64, True), (20, False)):
        plan = kv.KVLincRotary(kv.rotary_frequencies(channels), interleaved=interleaved)
        cache = kv.KVLincCache(1, 2, 1, 128)
        q = inputs(1, 2, 1, 3, "f16", False)[0]
        want = cache.rotary(plan, q)[0]
        bad = q.clone()
        bad[0, 0, 1, 3], bad[0, 1, 2, 100], bad[0, 1, 0, channels - 1] = float("inf"), float("nan"), float("nan")
        got = cache.rotary(plan, bad)[0]
        differ = {tuple(i) for i in torch.nonzero(~(got == want)).tolist()}
        pair = lambda c: {c, c ^ 1} if interleaved else {c, (c + channels // 2) % channels}
        assert differ == {(0, 0, 1, c) for c in pair(3)} | {(0, 1, 0, c) for c in pair(channels - 1)} | {(0, 1, 2, 100)}


def test_numbers_beyond_the_output_type():
    plan = kv.KVLincRotary([0.0] * 64)
    cache = kv.KVLincCache(1, 1, 1, 128)
    x = torch.full((1, 1, 1, 128), 1e6, device="cuda")
    x[..., 1] = -1e6
    y = cache.rotary(plan, x)[0]
    assert (y[..., 0] == float("inf")).all() and (y[..., 1] == float("-inf")).all()
    assert torch.equal(cache.rotary(plan, x, dtype=torch.float32)[0], x)  # (an angle of 0 leaves a number as it is)


def test_from_a_graph():
    plan = kv.KVLincRotary(kv.rotary_frequencies())
    cache = kv.KVLincCache(2, 8, 2, 1024)
    q, k, v = inputs(2, 8, 2, 3, "bf16", True)
    first = torch.zeros(2, dtype=torch.int32, device="cuda")
    outs, mine = ([torch.zeros(t.shape, dtype=torch.float16, device="cuda") for t in (q, k, v)] for _ in range(2))
    call = lambda o: cache.rotary(plan, q, k, v, first=first, q_out=o[0], k_out=o[1], v_out=o[2])

    def prepare(i):
        for t in (q, k, v):
            t.normal_()
        first.fill_(100 * i)
        cache.n_res.fill_(i)

    replayed(lambda: list(call(outs)), prepare, lambda: list(call(mine)))


@pytest.mark.parametrize("raw", [False, True])
def test_a_stream_of_the_callers(raw):
    plan = kv.KVLincRotary(kv.rotary_frequencies())
    cache = kv.KVLincCache(2, 8, 2, 1024)
    args = inputs(2, 8, 2, 50, "f16", True)
    want = cache.rotary(plan, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = cache.rotary(plan, *args, stream=side.cuda_stream if raw else side)
    del args
    filler = [torch.full((2, 8, 50, 128), 100.0, dtype=torch.float16, device="cuda") for _ in range(8)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(filler) == 8
