"""Eviction: which groups stay, that they stay bit for bit and in order, in place and into another cache; ties, numbers that are none, few and very many
groups, static caches, both widths, counters and offsets; what a decode sees afterwards."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from tests import bounded_reference as bounded
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_context_use import replayed
from tests.test_gpu_prompt_attention import filled

pytestmark = pytest.mark.gpu

BUFFERS = ("groups", "k_res", "v_res", "n_quant", "n_res")


def cache_of(B, H_q, H_kv, n_quant, n_res, room, bits=2, R=128, flags=0, seed=0):
    """A cache of random records (eviction moves them as they are)."""
    c = kv.KVLincCache(B, H_q, H_kv, 128 * room, R=R, bits=bits, flags=flags)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c.groups.random_(-2 ** 31, 2 ** 31 - 1, generator=gen)
    for t in (c.k_res, c.v_res):
        t.normal_(generator=gen)
    c.n_quant.copy_(torch.as_tensor(np.resize(n_quant, B)))
    c.n_res.copy_(torch.as_tensor(np.resize(n_res, B)))
    return c


def copy_of(c):
    d = kv.KVLincCache(c.B, c.H_q, c.H_kv, 128 * c.max_groups, R=c.R, bits=c.bits, flags=c.struct.flags)
    for name in BUFFERS:
        getattr(d, name).copy_(getattr(c, name))
    return d


def mass_of(c, seed=0, ties=False):
    m = torch.rand(c.B, c.H_kv, c.max_groups + 1, generator=torch.Generator().manual_seed(seed))
    return ((m * 4).floor() if ties else m).cuda()


def check(before, mass, after, mass_out, kept, offset_out, keep, limit, first, last, offset=None):
    """`before`: a copy of the cache as it was; `after`: the cache that the groups went to."""
    m, nq = mass.cpu().numpy(), before.n_quant.cpu().numpy()
    for b in range(before.B):
        n = -(-int(nq[b]) // 128)
        gone = 0
        for g in range(before.H_kv):
            want = bounded.stay(m[b, g], n, keep, limit, first, last)
            gone = n - len(want)
            if kept is not None:
                assert kept[b, g, :len(want)].tolist() == want, (b, g)
                assert (kept[b, g, len(want):] == -7).all()
            assert torch.equal(after.groups[b, g, :len(want)], before.groups[b, g, want]), (b, g)
            expect = torch.zeros(after.max_groups + 1, device="cuda")
            expect[:len(want)] = mass[b, g, want]
            expect[len(want)] = mass[b, g, n]
            assert torch.equal(mass_out[b, g].view(torch.int32), expect.view(torch.int32)), (b, g)  # (bit for bit: not numbers, too)
        assert after.n_quant[b].item() == nq[b] - 128 * gone and after.n_res[b].item() == before.n_res[b].item()
        if offset_out is not None:
            assert offset_out[b].item() == 128 * gone + (0 if offset is None else offset[b].item())
    assert torch.equal(after.k_res, before.k_res) and torch.equal(after.v_res.view(torch.int16), before.v_res.view(torch.int16))


def run_case(B, H_kv, n_quant, n_res, room, keep, limit=None, first=1, last=1, bits=2, R=128, flags=0, mass=None, ties=False, H_q=None, small=None, seed=0):
    limit = keep if limit is None else limit
    c = cache_of(B, H_q or H_kv, H_kv, n_quant, n_res, room, bits, R, flags, seed)
    mass = mass_of(c, seed, ties) if mass is None else mass
    before = copy_of(c)
    offset = torch.arange(B, dtype=torch.int32, device="cuda") * 1000
    # into a cache that has just the room
    to = cache_of(B, H_q or H_kv, H_kv, 0, 0, small or min(limit, room), bits, R, flags, seed + 1)
    kept = torch.full((B, H_kv, to.max_groups), -7, dtype=torch.int32, device="cuda")
    mass_out, offset_out = torch.full((B, H_kv, to.max_groups + 1), 5.0, device="cuda"), torch.full_like(offset, -1)
    was = mass.clone()
    assert c.evict(mass, keep, limit=limit, first=first, last=last, to=to, mass_out=mass_out, offset=offset, offset_out=offset_out, kept=kept) is to
    check(before, mass, to, mass_out, kept, offset_out, keep, limit, first, last, offset)
    assert torch.equal(was.view(torch.int32), mass.view(torch.int32))  # and the first one is as it was
    for name in BUFFERS:
        assert torch.equal(getattr(c, name).view(torch.int32), getattr(before, name).view(torch.int32)), name
    # in place
    kept = torch.full((B, H_kv, room), -7, dtype=torch.int32, device="cuda")
    moved, offset_out = mass.clone(), offset.clone()
    assert c.evict(moved, keep, limit=limit, first=first, last=last, offset=offset_out, kept=kept) is c
    check(before, mass, c, moved, kept, offset_out, keep, limit, first, last, offset)
    # in place, with no more than is needed
    d = copy_of(before)
    other = torch.full_like(mass, 5.0)
    d.evict(mass, keep, limit=limit, first=first, last=last, mass_out=other)
    for name in BUFFERS:
        assert torch.equal(getattr(c, name).view(torch.int32), getattr(d, name).view(torch.int32)), name
    assert torch.equal(other.view(torch.int32), moved.view(torch.int32))
    return c


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("groups, keep, first, last", [(1, 1, 0, 1), (2, 1, 0, 1), (3, 2, 1, 1), (9, 4, 0, 1), (9, 4, 1, 3), (9, 4, 3, 1), (9, 8, 1, 1), (17, 16, 1, 2),
                                                       (40, 5, 2, 2), (64, 16, 0, 16), (300, 33, 1, 4), (300, 299, 1, 4), (700, 512, 0, 1)])
def test_sizes(groups, keep, first, last, bits):
    run_case(2, 3, [128 * groups], [1, 128], groups + 1, keep, first=first, last=last, bits=bits, seed=groups)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("room", [63, 64, 65, 127, 255, 256, 257, 511, 512, 513, 1024])
def test_as_many_groups_as_a_wave_or_a_launch_selects_from_and_one_more_or_less(room, bits):
    for n, keep, first, last in ((room, room - 1, 0, 1), (room - 1, room // 2, 1, 2), (room, 2, 1, 1)):
        c = run_case(1, 2, [128 * n], [7], room, keep, first=first, last=last, bits=bits, seed=room)
        assert (c.split_done == 0).all()


@pytest.mark.parametrize("B, H_kv", [(1, 1), (1, 40), (70, 3), (3, 33)])
def test_counters_that_tell_who_writes_last_are_zero_again(B, H_kv):
    c = cache_of(B, H_kv, H_kv, [128 * n for n in (30, 11, 10, 3)], [9, 1], 30)
    before, mass = copy_of(c), mass_of(c)
    offset = torch.zeros(B, dtype=torch.int32, device="cuda")
    for i in range(3):  # (the second and third time there is nothing to drop)
        moved = mass.clone() if i == 0 else moved
        c.evict(moved, 8, limit=10, first=1, last=2, offset=offset)
        assert (c.split_done == 0).all()
        check(before, mass, c, moved, None, offset, 8, 10, 1, 2)


def test_into_another_cache_with_the_mass_in_place():
    c = cache_of(3, 2, 2, [128 * n for n in (30, 11, 12)], [9, 1], 30)
    mass, before = mass_of(c), copy_of(c)
    to = cache_of(3, 2, 2, 0, 0, 30, seed=1)
    moved, offset = mass.clone(), torch.zeros(3, dtype=torch.int32, device="cuda")
    assert c.evict(moved, 8, limit=11, first=1, last=2, to=to, mass_out=moved, offset=offset) is to
    check(before, mass, to, moved, None, offset, 8, 11, 1, 2)
    assert (to.split_done == 0).all() and torch.equal(c.n_quant, before.n_quant) and torch.equal(c.groups, before.groups)


@pytest.mark.parametrize("bits, groups, keep", [(2, 800, 700), (4, 420, 370), (2, 1100, 900)])
def test_many_bytes(bits, groups, keep):
    run_case(2, 8, [128 * groups, 128 * groups - 128], [5, 128], groups, keep, first=2, last=3, bits=bits)


def test_ragged_lengths_and_a_limit_above_what_is_kept():
    run_case(8, 2, [0, 128, 512, 640, 768, 1024, 2048, 0], [0, 5, 1, 128, 128, 30, 77, 9], 20, 5, limit=6, last=2)
    run_case(5, 1, [128 * n for n in (30, 29, 28, 2, 12)], [64], 30, 12, limit=28, first=0, last=3, small=40)


@pytest.mark.parametrize("groups", [5, 300, 1500])
def test_of_equal_masses_the_oldest_stay(groups):
    run_case(1, 4, [128 * groups], [3], groups, groups // 2, ties=True)
    run_case(1, 1, [128 * groups], [3], groups, groups // 2, mass=torch.zeros(1, 1, groups + 1, device="cuda"))


def test_numbers_of_every_kind():
    n = 40
    m = torch.rand(1, 2, n + 1, generator=torch.Generator().manual_seed(2)) - 0.5
    m[0, 0, [3, 9, 20]] = float("nan")
    m[0, 0, [4, 30]] = float("inf")
    m[0, 0, [5, 31]] = float("-inf")
    m[0, 0, [6, 7, 8]] = torch.tensor([0.0, -0.0, 0.0])
    m[0, 0, 10], m[0, 0, 11] = 1e-45, -1e-45
    m[0, 1] = float("nan")
    m[0, 1, 17] = float("-inf")
    for keep in (3, 10, 19, 20, 21, 22, 30, 36, 37, 38, 39):
        run_case(1, 2, [128 * n], [1], n, keep, mass=m.cuda())


def test_zeros_of_either_sign_are_equal():
    m = torch.zeros(1, 1, 10)
    m[0, 0, ::2] = -0.0
    c = run_case(1, 1, [9 * 128], [1], 9, 5, first=0, mass=m.cuda())
    assert c.n_quant.item() == 5 * 128


@pytest.mark.parametrize("n_quant, n_res, R", [(600, 20, 32), (129, 1, 128), (1000, 64, 64)])
def test_static_caches_with_a_partial_group(n_quant, n_res, R):
    run_case(2, 2, [n_quant, n_quant - 100], [n_res], 9, 2, R=R)


def test_sliding_values_and_shapes():
    run_case(3, 2, [1280, 128, 640], [7, 128, 1], 11, 4, flags=kv.KVLINC_FLAG_SLIDING_VALUES, H_q=14)
    run_case(100, 1, [128 * 5], [9], 6, 3, H_q=8)
    run_case(2, 32, [128 * 12], [9], 12, 7)


def test_very_many_groups():
    c = run_case(1, 1, [128 * 20000], [9], 20001, 9000, first=3, last=70)
    assert c.n_quant.item() == 128 * 9000


def test_a_cache_beyond_four_gigabytes():
    n = 250_000  # records of 17408 bytes: 4.35 GB
    c = kv.KVLincCache(1, 1, 1, 128 * n, bits=4)
    c.groups[0, 0, :, 0] = torch.arange(n, device="cuda")
    c.groups[0, 0, :, -1] = -torch.arange(n, device="cuda", dtype=torch.int32)
    c.n_quant.fill_(128 * n)
    m = c.new_mass()
    m[0, 0, n // 2:n // 2 + 1000] = 1.0
    m[0, 0, n - 3000:n - 1000] = 2.0
    to = kv.KVLincCache(1, 1, 1, 128 * 3001, bits=4)
    out = to.new_mass()
    want = torch.cat((torch.arange(n // 2, n // 2 + 1000), torch.arange(n - 3000, n - 1000), torch.tensor([n - 1]))).int().cuda()
    c.evict(m, 3001, first=0, to=to, mass_out=out)
    assert torch.equal(to.groups[0, 0, :, 0], want) and torch.equal(to.groups[0, 0, :, -1], -want)
    c.evict(m, 3001, first=0)
    assert torch.equal(c.groups[0, 0, :3001], to.groups[0, 0]) and c.n_quant.item() == 128 * 3001 and torch.equal(m[0, 0, :3002], out[0, 0])


def test_what_is_seen_afterwards():
    """The decode over the cache that is left is the softmax over the tokens that are left."""
    B, H_q, H_kv, lengths, keep = 2, 8, 2, [1500, 900], 4
    K, V, q, k_new, v_new = ref.inputs(1700, B, H_q, H_kv, lengths, 1)
    cache = filled(B, H_q, H_kv, K, V, 2048)
    mass = cache.new_mass()
    cache.decode_mass(to_dev(q[:, :, 0]), mass)
    kept = torch.zeros(B, H_kv, cache.max_groups, dtype=torch.int32, device="cuda")
    offset = torch.zeros(B, dtype=torch.int32, device="cuda")
    cache.evict(mass, keep, last=2, kept=kept, offset=offset)
    assert (cache.n_quant == 128 * keep).all() and offset.tolist() == [1408 - 512, 896 - 512]
    cache.append(to_dev(k_new), to_dev(v_new))
    out, seen = cache.decode(to_dev(q[:, :, 0])).cpu().numpy(), cache.decode_windowed(to_dev(q[:, :, 0]), 0).cpu().numpy()
    for b, n in enumerate(lengths):
        nq = (n - 1) // 128 * 128
        for g in range(H_kv):
            keys, values, _ = ref.tokens_of(K[b][g], V[b][g], nq)
            t = np.concatenate([np.arange(128 * j, 128 * j + 128) for j in kept[b, g, :keep].tolist()] + [np.arange(nq, n)])
            new_v = ref.tokens_of(k_new[b, g], v_new[b, g], 0)[1]
            keys, values = np.concatenate([keys[t], k_new[b, g].astype(np.float64)]), np.concatenate([values[t], new_v])
            for h in range(4 * g, 4 * g + 4):
                y, tol = ref.attend(q[b, h], keys, values, [len(keys) - 1])
                ref.check_rows(out[b, h][None], y, tol, (b, h))
                ref.check_rows(seen[b, h][None], y, tol, (b, h))


def test_in_place_from_a_graph():
    """One group over the budget, then none, then many: a captured call goes by the counters it finds."""
    c, d = (cache_of(3, 4, 2, [128 * 9], [5], 16, seed=4) for _ in range(2))
    source, m0 = copy_of(c), mass_of(c, 9)
    mass, other = m0.clone(), m0.clone()
    offset = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2)]

    def prepare(i):
        for x in (c, d):
            for name in BUFFERS:
                getattr(x, name).copy_(getattr(source, name))
            x.n_quant.copy_(128 * torch.tensor([[9, 8, 16], [0, 1, 7], [16, 16, 2], [8, 9, 10], [9, 9, 9], [12, 3, 16]][i]))
        m0.uniform_()
        mass.copy_(m0)
        other.copy_(m0)

    def call(x, m, o):
        x.evict(m, 8, first=1, last=2, offset=o)
        return [t.view(torch.int16) for t in (x.groups, x.n_quant, m, o)]

    # (replayed() spoils the outputs it is given ahead of a replay: copies of them)
    outs = [torch.empty_like(t) for t in (c.groups, c.n_quant, mass, offset[0])]

    def capture():
        call(c, mass, offset[0])
        for dst, src in zip(outs, (c.groups, c.n_quant, mass, offset[0])):
            dst.copy_(src)
        return [t.view(torch.int16) for t in outs]

    replayed(capture, prepare, lambda: call(d, other, offset[1]))


@pytest.mark.parametrize("raw", [False, True])
def test_a_stream_of_the_callers(raw):
    c = cache_of(2, 4, 2, [128 * 30], [5], 31)
    mass = mass_of(c)
    want, mass_want = copy_of(c), mass.clone()
    want.evict(mass_want, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    to = kv.KVLincCache(2, 4, 2, 128 * 9)
    out = to.new_mass()
    side.wait_stream(torch.cuda.current_stream())
    c.evict(mass, 9, to=to, mass_out=out, stream=side.cuda_stream if raw else side)
    del mass
    filler = [torch.full((2, 2, 32), 100.0, device="cuda") for _ in range(8)]
    side.synchronize()
    assert torch.equal(to.groups, want.groups[:, :, :9]) and torch.equal(out, mass_want[:, :, :10]) and len(filler) == 8
