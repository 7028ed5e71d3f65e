"""The calls of kvlinc_context.h as a model would make them: one after the other over a growing cache, from graphs, on other streams, at the
ends of their ranges."""
import numpy as np
import pytest
import torch

import kvlinc_synth as synth
import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev
from tests.test_gpu_prompt_attention import filled, run_case

pytestmark = pytest.mark.gpu


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def inputs(B, H_q, H_kv, T, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(B, h, T, 128, generator=gen).half().cuda() for h in (H_q, H_kv, H_kv))


# ---- one after the other ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits, corr, sliding", [(2, False, False), (4, False, True), (2, True, False), (4, True, False), (2, True, True)])
def test_a_prompt_chunks_drafts_and_decoding(bits, corr, sliding):
    config, B, H_q, H_kv, gq = 970, 2, 8, 2, 4
    most = 900
    K = np.stack([[synth.keys(config, b, g, most) for g in range(H_kv)] for b in range(B)])
    V = np.stack([[synth.values(config, b, g, most) for g in range(H_kv)] for b in range(B)])
    Wq, Wk = (synth.adapters_q(config, H_q), synth.adapters_k(config, H_kv)) if corr else (None, None)
    cache = kv.KVLincCache(B, H_q, H_kv, most, Wq=None if Wq is None else to_dev(Wq), Wk=None if Wk is None else to_dev(Wk), bits=bits,
                           flags=kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0)
    held = [0, 0]

    def rows_of(T, rows, x):
        out = np.zeros((B, H_kv, T, 128), np.float16)
        for b in range(B):
            out[b, :, :rows[b]] = x[b, :, held[b]:held[b] + rows[b]]
        return out

    def expect(b, h, q, extra, positions, window=0, sinks=0):
        n, g = held[b], h // gq
        keys, values, oc = ref.tokens_of(K[b, g, :n], V[b, g, :n], o_cache.window_split(n)[0] if n else 0, bits, sliding, Wk[g] if corr else None)
        keys = np.concatenate([keys, K[b, g, n:n + extra].astype(np.float64)])
        values = np.concatenate([values, V[b, g, n:n + extra].astype(np.float64)])
        return ref.attend(q, keys, values, positions, window, sinks, oc, Wq[h] if corr else None)

    def attend(step, T, rows, window=0, sinks=0):
        q = np.stack([np.stack([synth.queries(config, b, H_q, step=step + i) for i in range(T)], 1) for b in range(B)])
        n_new = None if rows == [T] * B else to_dev(np.asarray(rows, np.int32))
        k, v = rows_of(T, rows, K), rows_of(T, rows, V)
        got = cache.prompt_attention(to_dev(q), to_dev(k), to_dev(v), n_new=n_new, window=window, sinks=sinks).cpu().numpy()
        for b in range(B):
            assert (got[b, :, rows[b]:] == 0).all()
            for h in range(H_q):
                y, tol = expect(b, h, q[b, h, :rows[b]], rows[b], held[b] + np.arange(rows[b]), window, sinks)
                ref.check_rows(got[b, h, :rows[b]], y, tol, (step, b, h))

    def append(T, rows):
        cache.append(to_dev(rows_of(T, rows, K)), to_dev(rows_of(T, rows, V)), n_new=to_dev(np.asarray(rows, np.int32)))
        for b in range(B):
            held[b] += rows[b]

    attend(0, 300, [300, 170])      # the prompt, from an empty cache
    append(300, [300, 170])
    attend(400, 70, [70, 70])       # a chunk
    append(70, [70, 70])
    for step in range(3):           # drafts: some of them kept
        attend(500 + 10 * step, 5, [5, 5])
        append(5, [3 - step, step])
    if not corr:
        attend(600, 40, [40, 11], window=100, sinks=2)
    for step in range(3):           # tokens one by one
        append(1, [1, 1])
        q = np.stack([synth.queries(config, b, H_q, step=700 + step) for b in range(B)])
        for window in (0,) if corr else (0, 64):
            got = (cache.decode_windowed(to_dev(q), window, sinks=1) if not corr else cache.decode(to_dev(q))).cpu().numpy()
            for b in range(B):
                for h in range(H_q):
                    y, tol = expect(b, h, q[b, h][None], 0, [held[b] - 1], window, 1)
                    d = np.linalg.norm(got[b, h] - y[0])
                    assert d <= max(tol[0], 2e-3 * np.linalg.norm(y[0])), (step, b, h, d, tol)
    assert cache.n_quant.tolist() == [o_cache.window_split(n)[0] for n in held] and cache.status.item() == 0
    k, v = cache.read(T=max(held), dtype=torch.float32)
    for b in range(B):
        n = held[b]
        for g in range(H_kv):
            keys, values, _ = ref.tokens_of(K[b, g, :n], V[b, g, :n], o_cache.window_split(n)[0], bits, sliding)
            assert np.abs(k[b, g, :n].cpu().numpy() - keys).max() <= 2.0 ** -20 * np.abs(keys).max()
            assert np.abs(v[b, g, :n].cpu().numpy() - values).max() <= 2.0 ** -20 * np.linalg.norm(values, axis=1).max()
        assert (k[b, :, n:] == 0).all() and (v[b, :, n:] == 0).all()


def test_decoding_is_what_it_was_after_these_calls():
    K, V, _, _, _ = ref.inputs(971, 2, 8, 2, [3000, 700], 1)
    cache = filled(2, 8, 2, K, V, 4096)
    q1 = torch.randn(2, 8, 128, device="cuda").half()
    want = cache.decode(q1)
    for T in (1, 5, 40, 300):
        cache.prompt_attention(*inputs(2, 8, 2, T))
        cache.decode_windowed(q1, 2000, sinks=4)
        cache.read(T=100)
        assert same(cache.decode(q1), want)


def test_workspaces_of_different_sizes():
    K, V, _, _, _ = ref.inputs(972, 1, 8, 1, [2000], 1)
    cache = filled(1, 8, 1, K, V, 2304)
    sizes = (2, 300, 60, 2, 900, 1)
    calls = [inputs(1, 8, 1, T, T) for T in sizes]
    got = [cache.prompt_attention(*c) for c in calls]
    for c, g in zip(calls, got):
        assert same(filled(1, 8, 1, K, V, 2304).prompt_attention(*c), g)


def test_scratch_that_is_outgrown_is_given_back():
    cache = kv.KVLincCache(1, 8, 2, 1 << 16)
    args = inputs(1, 8, 2, 300)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for bound in range(1 << 12, 1 << 16, 1 << 12):  # (room for the dequantized tokens of the bound)
        cache.prompt_attention(*args, max_context=bound, out=torch.empty_like(args[0]))
    need = kv.kvlinc_prompt_workspace_bytes(cache, 300, max_context=15 << 12)
    assert need > 2 * 15 * 4096 * 512 and torch.cuda.memory_allocated() - before < need + (1 << 22)


# ---- graphs ----------------------------------------------------------------------------------------------------------------------

def replayed(capture, prepare, eager, replays=6):
    """The outputs of a captured call against the eager one's, over several replays with other work between them."""
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = capture()
    for i in range(replays):
        prepare(i)
        want = [t.clone() for t in eager()]
        for t in outs:
            t.fill_(3.0)
        scratch = torch.randn(512, 512, device="cuda")
        (scratch @ scratch).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(outs, want)), i
    return graph


@pytest.mark.parametrize("T, corr, window", [(1, True, 0), (4, False, 200), (6, True, 0), (40, False, 0), (40, True, 0), (300, False, 500), (300, True, 0)])
def test_prompt_attention_from_a_graph(T, corr, window):
    config = 973
    K, V, _, _, _ = ref.inputs(config, 2, 8, 2, [2000, 300], 1)
    Wq, Wk = (to_dev(synth.adapters_q(config, 8)), to_dev(synth.adapters_k(config, 2))) if corr else (None, None)
    cache = filled(2, 8, 2, K, V, 4096, Wq=Wq, Wk=Wk)
    q, k, v = inputs(2, 8, 2, T)
    n_new = torch.tensor([T, max(1, T // 2)], dtype=torch.int32, device="cuda")
    out, mine = torch.zeros_like(q), torch.zeros_like(q)

    def prepare(i):
        for dst, src in zip((q, k, v), inputs(2, 8, 2, T, 50 + i)):
            dst.copy_(src)
        if i == 3:  # another context: the graph reads the counters as they are
            cache.append(k[:, :, :1].contiguous(), v[:, :, :1].contiguous())
        mine.fill_(3.0)

    replayed(lambda: [cache.prompt_attention(q, k, v, n_new=n_new, window=window, sinks=3, out=out)], prepare,
             lambda: [cache.prompt_attention(q, k, v, n_new=n_new, window=window, sinks=3, out=mine)])
    assert int(cache.split_done.abs().sum()) == 0


def test_windowed_decode_and_reading_from_a_graph():
    K, V, _, _, _ = ref.inputs(974, 2, 8, 2, [3000, 700], 1)
    cache = filled(2, 8, 2, K, V, 4096)
    q = torch.zeros(2, 8, 128, dtype=torch.float16, device="cuda")
    first = torch.zeros(2, dtype=torch.int32, device="cuda")
    row = torch.zeros(2, 2, 1, 128, dtype=torch.float16, device="cuda")
    bufs = [torch.zeros(2, 2, 70, 128, dtype=torch.float16, device="cuda") for _ in range(4)]
    out, mine = torch.zeros_like(q), torch.zeros_like(q)

    def call(out, k, v):
        cache.decode_windowed(q, 2100, sinks=5, out=out)
        cache.read(first=first, k_out=k, v_out=v)
        return [out, k, v]

    def prepare(i):
        q.normal_()
        row.normal_()
        cache.append(row, row)
        first.copy_(torch.tensor([100 * i, 200 + i], dtype=torch.int32))
        for t in bufs:
            t.fill_(3.0)

    replayed(lambda: call(out, *bufs[:2]), prepare, lambda: call(mine, *bufs[2:]))


def test_two_graphs_that_share_a_workspace():
    K, V, _, _, _ = ref.inputs(975, 1, 8, 2, [2500], 1)
    cache = filled(1, 8, 2, K, V, 4096)
    sizes = (5, 40)
    args = [inputs(1, 8, 2, T, T) for T in sizes]
    outs = [torch.zeros_like(a[0]) for a in args]
    graphs = []
    for a, o in zip(args, outs):  # (the second needs more scratch than the first)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.prompt_attention(*a, out=o)
        graphs.append(g)
    want = [cache.prompt_attention(*a) for a in args]
    for turn in range(4):
        for t in outs:
            t.fill_(3.0)
        for g in graphs if turn % 2 else reversed(graphs):
            g.replay()
        cache.prompt_attention(*inputs(1, 8, 2, 300))  # (and eager work takes still more)
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))


# ---- streams ---------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("raw", [False, True])
def test_a_stream_of_the_callers(raw):
    K, V, _, _, _ = ref.inputs(976, 2, 8, 2, [2000, 300], 1)
    cache = filled(2, 8, 2, K, V, 2304)
    q1 = torch.randn(2, 8, 128, device="cuda").half()
    side = torch.cuda.Stream()
    handle = side.cuda_stream if raw else side
    for T in (3, 40, 300):
        want = cache.prompt_attention(*inputs(2, 8, 2, T)), cache.decode_windowed(q1, 900), *cache.read(T=50)
        args = inputs(2, 8, 2, T)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)  # (the call starts some milliseconds from now)
        got = [cache.prompt_attention(*args, stream=handle)]
        del args
        filler = [torch.full((2, 8, T, 128), 100.0, dtype=torch.float16, device="cuda") for _ in range(8)]  # what was freed is not theirs yet
        got += [cache.decode_windowed(q1, 900, stream=handle), *cache.read(T=50, stream=handle)]
        torch.cuda.current_stream().wait_stream(side)
        assert all(same(a, b) for a, b in zip(got, want))
        del filler


def test_a_cache_that_is_dropped_while_a_stream_reads_it():
    K, V, q, k_new, v_new = ref.inputs(995, 1, 8, 2, [2000], 4)
    args = [to_dev(x) for x in (q, k_new, v_new)]
    want = filled(1, 8, 2, K, V, 2304).prompt_attention(*args)
    cache, side = filled(1, 8, 2, K, V, 2304), torch.cuda.Stream()
    size = cache.groups.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = cache.prompt_attention(*args, stream=side)
    del cache
    filler = [torch.full((size,), -1, dtype=torch.int32, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert same(got, want)
    del filler


def test_two_caches_on_two_streams():
    caches, args, want = [], [], []
    for i in range(2):
        K, V, _, _, _ = ref.inputs(977 + i, 1, 8, 2, [3000], 1)
        caches.append(filled(1, 8, 2, K, V, 4096))
        args.append([inputs(1, 8, 2, T, 10 * i + T) for T in (4, 40, 300)])
        want.append([caches[i].prompt_attention(*a) for a in args[i]] + [caches[i].decode_windowed(args[i][0][0][:, :, 0].contiguous(), 2500)])
    ones = [a[0][0][:, :, 0].contiguous() for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(5):
        got = [[], []]
        for k in range(4):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    got[i].append(caches[i].prompt_attention(*args[i][k]) if k < 3 else caches[i].decode_windowed(ones[i], 2500))
        torch.cuda.synchronize()
        assert all(same(a, b) for i in range(2) for a, b in zip(got[i], want[i]))


def test_windowed_decode_over_its_own_queries():
    K, V, _, _, _ = ref.inputs(979, 2, 16, 2, [4000, 100], 1)
    cache = filled(2, 16, 2, K, V, 4096)
    q = torch.randn(2, 16, 128, device="cuda").half()
    want = cache.decode_windowed(q, 3000)
    for _ in range(4):
        mine = q.clone()
        assert cache.decode_windowed(mine, 3000, out=mine) is mine and same(mine, want)
    with pytest.raises(kv.KVLincError):
        x = inputs(2, 16, 2, 3)
        cache.prompt_attention(*x, out=x[0])


# ---- the ends of the ranges ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [4, 5, 8, 9, 16, 17, 32, 33, 48, 49, 64, 65, 256, 257, 511, 512, 513, 1023, 1024])
def test_numbers_of_rows_where_the_work_is_laid_out_anew(rows):
    run_case(980, 1, 1, [333], [rows])


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("window, sinks", [(300, 5), (64, 64), (65, 1), (1, 200), (700, 0)])
def test_sinks_apart_from_the_window_and_many_rows(window, sinks, bits):
    run_case(981, 4, 1, [2000, 350], [270, 260], bits, window, sinks)


@pytest.mark.parametrize("lengths, rows, H_q, H_kv", [([5000], [1], 8, 2), ([5000, 40], [4, 4], 4, 1), ([6000], [6], 8, 2), ([5000], [40], 4, 1),
                                                       ([5000, 900], [40, 3], 8, 8), ([4500], [260], 8, 1)])
@pytest.mark.parametrize("corr", [False, True])
def test_long_contexts_in_splits(lengths, rows, H_q, H_kv, corr):
    run_case(982, H_q, H_kv, lengths, rows, corr=corr)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("window, sinks, corr, sliding, keep", [(0, 0, False, False, 0), (100, 3, False, False, 0), (1, 200, False, True, 0), (700, 1, False, False, 60),
                                                                (0, 0, True, False, 0), (0, 0, True, True, 0), (0, 0, False, False, 32)])
def test_two_blocks_of_rows(window, sinks, corr, sliding, keep, bits):
    run_case(992, 8, 2, [900, 130, 0, 385], [128, 100, 65, 3], bits, window, sinks, corr=corr, sliding=sliding, keep=keep, R=64 if keep else 128)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("T", [3, 40, 300])
def test_keys_of_different_magnitudes(T, bits):
    # channels from 2^-10 to 2^10 of one another, and queries that even them out: every scale of the parts that the rounding of a key leaves
    B, H_q, H_kv, n = 1, 4, 1, 400
    K, V, q, k_new, v_new = ref.inputs(993, B, H_q, H_kv, [n], T)
    gain = 2.0 ** np.random.default_rng(3).integers(-10, 11, 128)
    K = [[(K[0][0].astype(np.float32) * gain).astype(np.float16)]]
    k_new, q = (k_new.astype(np.float32) * gain).astype(np.float16), (q.astype(np.float32) / gain).astype(np.float16)
    cache = filled(B, H_q, H_kv, K, V, 512, bits)
    assert cache.status.item() == 0
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0], bits)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    for h in range(H_q):
        y, tol = ref.attend(q[0, h], keys, values, n + np.arange(T))
        ref.check_rows(got[0, h], y, tol, h)


@pytest.mark.parametrize("bits", [2, 4])
@pytest.mark.parametrize("H_q, H_kv, T", [(8, 2, 4), (8, 2, 40), (8, 2, 150)])
def test_what_the_roundings_come_to(H_q, H_kv, T, bits):
    # All rows together, as norms of independent roundings.  One is uniform in half a step, 2^-11 / sqrt(12) = 1.4e-4 relative where a binade
    # starts and half of that where it ends: the output's, the weights', the values' (of s |code|, up to twice the value: counted as two), and a
    # tenth of what binary16 keys would cost the scores, 2^-12 / sqrt(3) * sqrt(380 / 128) = 2.4e-4.  sqrt(1 + 1 + 4) * 1.4e-4 = 3.4e-4 at the most,
    # and 1.4 times that for the rows that few tokens decide: their roundings are no average.  Binary16 keys alone: 8e-4.
    B, n = 2, 1500
    K, V, q, k_new, v_new = ref.inputs(994, B, H_q, H_kv, [n] * B, T)
    cache = filled(B, H_q, H_kv, K, V, 2048, bits)
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    num = den = 0.0
    for b in range(B):
        for g in range(H_kv):
            keys, values, _ = ref.tokens_of(K[b][g], V[b][g], o_cache.window_split(n)[0], bits)
            keys, values = np.concatenate([keys, k_new[b, g].astype(np.float64)]), np.concatenate([values, v_new[b, g].astype(np.float64)])
            for h in range(g * (H_q // H_kv), (g + 1) * (H_q // H_kv)):
                y, tol = ref.attend(q[b, h], keys, values, n + np.arange(T))
                d2, y2 = ref.check_rows(got[b, h], y, tol, (b, h))
                num, den = num + d2, den + y2
    assert (num / den) ** 0.5 <= 4.8e-4, (num / den) ** 0.5


@pytest.mark.parametrize("pairs", [3, 8, 16, 24])
def test_blocks_of_rows_of_several_pairs(pairs):
    run_case(983, pairs, pairs, [200, 0, 70], [520, 260, 40])
    run_case(984, pairs, pairs, [200], [1030])


@pytest.mark.parametrize("T", [3, 40, 300])
def test_the_largest_keys(T):
    # keys of +-65504, queries of some 2^-15 (subnormal steps and all): scores of a few units.  A dequantized key beyond 65504 is held as
    # that, 2^-11 of it off at most: the bound's rounding of keys.
    B, H_q, H_kv, n = 1, 4, 1, 300
    K, V, q, k_new, v_new = ref.inputs(985, B, H_q, H_kv, [n], T)
    K = [[(np.sign(K[0][0]) * 65504).astype(np.float16)]]
    k_new = (np.sign(k_new) * 65504).astype(np.float16)
    q = (np.clip(q.astype(np.float32), -3, 3) * 2.0 ** -16).astype(np.float16)
    K[0][0][K[0][0] == 0] = 65504
    for bits in (2, 4):
        cache = filled(B, H_q, H_kv, K, V, 512, bits)
        assert cache.status.item() == 0
        got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
        keys, values, _ = ref.tokens_of(K[0][0], V[0][0], 256, bits)
        keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
        for h in range(H_q):
            y, tol = ref.attend(q[0, h], keys, values, n + np.arange(T))
            ref.check_rows(got[0, h], y, tol, h)


@pytest.mark.parametrize("n", [0, 300])
@pytest.mark.parametrize("T", [3, 40, 300])
def test_the_largest_new_values(n, T):
    B, H_q, H_kv = 1, 4, 1
    K, V, q, k_new, v_new = ref.inputs(986, B, H_q, H_kv, [n], T)
    v_new = np.where(v_new < 0, -65504, 65504).astype(np.float16)
    v_new[:, :, :, 5] = 65504  # a column whose mean is the largest number
    cache = filled(B, H_q, H_kv, K, V, 512)
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], 256 if n else 0)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    for h in range(H_q):
        y, tol = ref.attend(q[0, h], keys, values, n + np.arange(T))
        ref.check_rows(got[0, h], y, tol, h)


def one_winner(q, keys, values, positions, window=0, sinks=0):
    """Rows whose largest score is ahead of all others by more than the scores' errors and 30: the values of those tokens (None elsewhere);
    equal keys share."""
    s = q.astype(np.float64) @ keys.T / np.sqrt(128.0)
    t, p = np.arange(len(keys)), np.asarray(positions)[:, None]
    seen = (t <= p) & ((window == 0) | (p - t < window) | (t < sinks))
    s = np.where(seen, s, -np.inf)
    d = (2.0 ** -11 + 2.0 ** -14) * (np.abs(q.astype(np.float64)) @ np.abs(keys).T).max(1) / np.sqrt(128.0)
    out = []
    for i in range(len(q)):
        best = s[i] == s[i].max()
        rest = s[i][~best & np.isfinite(s[i])]
        out.append(values[best].mean(0) if len(rest) == 0 or s[i].max() - rest.max() > 2 * d[i] + 30 else None)
    return out


@pytest.mark.parametrize("gain", [30.0, 1000.0, 20000.0])
@pytest.mark.parametrize("T", [4, 40, 300])
def test_scores_of_any_size_pick_their_token(T, gain):
    # Queries along one key each, scores up to some 10^10: the softmax is that token's value, or the mean of two whose keys are equal.  Output:
    # weights and values rounded once each, and the output, 2^-11 of the norms.
    B, H_q, H_kv, n = 1, 4, 1, 300
    K, V, q, k_new, v_new = ref.inputs(987, B, H_q, H_kv, [n], T)
    rng = np.random.default_rng(5)
    K = [[np.clip(K[0][0].astype(np.float32) * gain, -60000, 60000).astype(np.float16)]]
    k_new = np.clip(k_new.astype(np.float32) * gain, -60000, 60000).astype(np.float16)
    if T > 4:
        k_new[0, 0, 3] = k_new[0, 0, 2]  # equal keys, different values: equal weights at any score
    cache = filled(B, H_q, H_kv, K, V, 512)
    assert cache.status.item() == 0
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], 256)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    for h in range(H_q):
        for i in range(T):
            target = n + 2 if i % 3 == 0 and i > 3 else int(rng.integers(0, n + i + 1))
            q[0, h, i] = np.clip(keys[target], -60000, 60000).astype(np.float16)
    got = cache.prompt_attention(to_dev(q), to_dev(k_new), to_dev(v_new)).cpu().numpy()
    assert np.isfinite(got).all()
    checked = 0
    for h in range(H_q):
        for i, want in enumerate(one_winner(q[0, h], keys, values, n + np.arange(T))):
            if want is not None:
                checked += 1
                spread = np.linalg.norm(values, axis=1).max()
                assert np.linalg.norm(got[0, h, i] - want) <= 3 * ref.HALF_STEP * spread + 1e-6, (h, i)
    assert checked > T


# ---- offsets beyond 32 bits ------------------------------------------------------------------------------------------------------

def test_records_beyond_4_gb():
    B, H_q, H_kv, room = 1, 4, 2, 300000 * 128  # 2.7 GB of records a KV head
    K, V, q, k_new, v_new = ref.inputs(988, B, H_q, H_kv, [400], 300)
    big, small = (filled(B, H_q, H_kv, K, V, r) for r in (room, 768))
    assert big.groups.numel() * 4 > 1 << 32
    for T in (3, 40, 300):
        args = [np.ascontiguousarray(x[:, :, :T]) for x in (q, k_new, v_new)]
        a, b = (c.prompt_attention(*(to_dev(x) for x in args), max_context=400) for c in (big, small))
        assert same(a, b)
    one = to_dev(q[:, :, 0])
    assert same(big.decode_windowed(one, 300, max_context=400), small.decode_windowed(one, 300, max_context=400))
    assert all(same(a, b) for a, b in zip(big.read(T=400), small.read(T=400)))


def test_rows_beyond_4_gb():
    # the last of 130 sequences has rows, and a context, the others none; 131072 rows a head: 4.4 GB a tensor
    B, T, n, rows = 130, 131072, 300, 700
    K, V, q, k_new, v_new = ref.inputs(989, 1, 1, 1, [n], rows)
    cache = kv.KVLincCache(B, 1, 1, 512)
    small = filled(1, 1, 1, K, V, 512)
    for name in ("groups", "k_res", "v_res", "n_quant", "n_res"):
        getattr(cache, name)[B - 1:].copy_(getattr(small, name))
    big = [torch.empty(B, 1, T, 128, dtype=torch.float16, device="cuda") for _ in range(4)]
    for dst, src in zip(big, (q, k_new, v_new)):
        dst[B - 1, :, :rows] = to_dev(src[0])
    big[3][B - 1] = 7.0
    n_new = torch.zeros(B, dtype=torch.int32, device="cuda")
    n_new[B - 1] = rows
    got = cache.prompt_attention(*big[:3], n_new=n_new, out=big[3], max_context=n)
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], 256)
    keys, values = np.concatenate([keys, k_new[0, 0].astype(np.float64)]), np.concatenate([values, v_new[0, 0].astype(np.float64)])
    y, tol = ref.attend(q[0, 0], keys, values, n + np.arange(rows))
    ref.check_rows(got[B - 1, 0, :rows].cpu().numpy(), y, tol, "rows")
    assert bool((got[B - 1, 0, rows:] == 7.0).all())
    # read back into rows as far apart
    big[0][B - 1], big[1][B - 1] = 3.0, 3.0
    cache.read(k_out=big[0], v_out=big[1])
    for t, want in zip(big, small.read(T=n)):
        assert same(t[B - 1, :, :n], want[0]) and bool((t[B - 1, :, n:] == 3.0).all())


@pytest.mark.parametrize("gain", [1000.0, 4000.0, 20000.0])
def test_windowed_scores_of_any_size_pick_their_token(gain):
    B, H_q, H_kv, n = 1, 4, 1, 700
    K, V, _, _, _ = ref.inputs(991, B, H_q, H_kv, [n], 1)
    K = [[np.clip(K[0][0].astype(np.float32) * gain, -60000, 60000).astype(np.float16)]]
    cache = filled(B, H_q, H_kv, K, V, 768)
    assert cache.status.item() == 0
    keys, values, _ = ref.tokens_of(K[0][0], V[0][0], o_cache.window_split(n)[0])
    rng, checked = np.random.default_rng(6), 0
    for _ in range(40):
        q = np.stack([np.clip(keys[int(rng.integers(0, n))], -60000, 60000).astype(np.float16) for _ in range(H_q)])
        window, sinks = int(rng.integers(0, 2)) * 400, 130
        got = cache.decode_windowed(to_dev(q[None]), window, sinks=sinks).cpu().numpy()[0]
        assert np.isfinite(got).all()
        for h in range(H_q):
            want = one_winner(q[h][None], keys, values, [n - 1], window, sinks)[0]
            if want is not None:
                checked += 1
                assert np.linalg.norm(got[h] - want) <= 3 * ref.HALF_STEP * np.linalg.norm(values, axis=1).max() + 1e-6
    assert checked > 40
