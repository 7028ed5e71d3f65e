"""Long generation in a bounded cache, as a program runs it: a prompt rotated, attended and appended, its last rows' attention weight, eviction into a smaller
cache, and generated tokens that are rotated, appended and attended while groups are evicted, eagerly and from a graph, against a model of it on the host."""
import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv
from oracle import kvcache as o_cache
from tests import bounded_reference as bounded
from tests import context_reference as ref
from tests.kvlinc_testlib import to_dev

pytestmark = pytest.mark.gpu

B, H_q, H_kv, GQ = 2, 4, 2, 2


class Host:
    """The tokens of one (sequence, KV head) that are left: fp16 rows as they were appended, in groups of 128, the window behind them."""

    def __init__(self, bits):
        self.bits, self.groups, self.window, self.raw_values = bits, [], [], None

    def append(self, k, v):
        if len(self.window) == 128:
            K, V = (np.stack([row[i] for row in self.window]) for i in range(2))
            self.groups.append(ref.tokens_of(K, V, 128, self.bits)[:2] + (o_cache.build_cache(K, V, 128, bits=self.bits),))
            self.raw_values = ref.tokens_of(K, V, 0, self.bits)[1]  # of the newest group, as the window had them
            self.window = []
        self.window.append((k, v))

    def tokens(self):
        """keys, values, slots, sizes"""
        K, V = (np.stack([row[i] for row in self.window]) for i in range(2))
        win = ref.tokens_of(K, V, 0, self.bits)[:2]
        levels = 2 ** self.bits - 1
        size = [np.tile(levels * c["k_scale"][0].astype(np.float64) + np.abs(c["k_zero"][0].astype(np.float64)), (128, 1)) for _, _, c in self.groups]
        keys, values = (np.concatenate([g[i] for g in self.groups] + [win[i]]) for i in range(2))
        slots = np.concatenate([np.full(128, j) for j in range(len(self.groups))] + [np.full(len(self.window), len(self.groups))]).astype(int)
        return keys, values, slots, np.concatenate(size + [np.abs(win[0])])

    def evict(self, mass, keep, limit, first, last):
        stays = bounded.stay(mass, len(self.groups), keep, limit, first, last)
        gone = len(self.groups) - len(stays)
        self.groups = [self.groups[j] for j in stays]
        return gone


def projected(step, T):
    """What a projection gives, [B, T, heads, 128] in bfloat16: seeded by the step."""
    gen = torch.Generator().manual_seed(1000 + step)
    x = torch.randn(B, T, H_q + 2 * H_kv, 128, generator=gen)
    x[:, :, H_q:H_q + H_kv, [3, 50, 77, 100]] *= 8.0
    return x.bfloat16().cuda().transpose(1, 2)


@pytest.mark.parametrize("bits, sliding, graph", [(2, False, False), (4, False, True), (2, True, True)])
def test_a_prompt_and_generation(bits, sliding, graph):
    lengths, T, keep, limit, first, last, steps, seen_rows = [1100, 700], 1100, 4, 5, 1, 1, 300, 20
    flags = kv.KVLINC_FLAG_SLIDING_VALUES if sliding else 0
    plan = kv.KVLincRotary(kv.rotary_frequencies(64, base=500000.0, scaling="parts", factor=4.0, original=512), magnitude=1.1)
    freq = plan.freq.cpu().numpy()
    ints = lambda a: to_dev(np.asarray(a, np.int32))
    prompts, cache = kv.KVLincCache(B, H_q, H_kv, 2048, bits=bits, flags=flags), kv.KVLincCache(B, H_q, H_kv, 128 * (limit + 1), bits=bits, flags=flags)
    host = [[Host(bits) for _ in range(H_kv)] for _ in range(B)]

    # ---- the prompt ----
    x = projected(0, T)
    parts = x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:]
    n_new = ints(lengths)
    q, k, v = prompts.rotary(plan, *parts, n_new=n_new)
    for got, raw, turned in zip((q, k, v), parts, (True, True, False)):
        for b, n in enumerate(lengths):
            y = raw[b, :, :n].double().cpu().numpy()
            y, off = bounded.rotated(y, np.arange(n), freq, False, 1.1) if turned else (y, 0.0)
            assert (np.abs(got[b, :, :n].double().cpu().numpy() - y) <= off + bounded.rounding(y, "f16")).all()
    out = prompts.prompt_attention(q, k, v, n_new=n_new)
    assert torch.isfinite(out).all()
    prompts.append(k, v, n_new=n_new)
    k_host, v_host = k.cpu().numpy(), v.cpu().numpy()
    for b in range(B):
        for g in range(H_kv):
            for t in range(lengths[b]):
                host[b][g].append(k_host[b, g, t], v_host[b, g, t])
    newest = torch.stack([q[b, :, n - seen_rows:n] for b, n in enumerate(lengths)])
    mass = prompts.attention_mass(newest)

    def accumulate(rows, got, before):
        """Masses of all pairs after rows [B, H_q, r, 128] of the newest tokens, against the host's."""
        got = got.cpu().numpy()
        for b in range(B):
            for g in range(H_kv):
                h = host[b][g]
                keys, _, slots, size = h.tokens()
                x = rows[b, g * GQ:(g + 1) * GQ].reshape(-1, 128)
                r = rows.shape[2]
                fresh, off = bounded.weights(x, keys, np.tile(len(keys) - r + np.arange(r), GQ), slots, len(h.groups) + 1, size)
                bounded.check_mass(got[b, g, :len(h.groups) + 1], before[b, g, :len(h.groups) + 1], 1.0, fresh, off, (b, g))
                assert (got[b, g, len(h.groups) + 1:] == 0).all()

    accumulate(newest.cpu().numpy(), mass, np.zeros(mass.shape))
    small, offset = cache.new_mass(), torch.zeros(B, dtype=torch.int32, device="cuda")
    kept = torch.zeros(B, H_kv, cache.max_groups, dtype=torch.int32, device="cuda")
    prompts.evict(mass, keep, limit=limit, first=first, last=last, to=cache, mass_out=small, offset=None, offset_out=offset, kept=kept)
    gone = np.zeros(B, int)

    def evicted(before):
        """The host's eviction by the masses before it; offsets, counters."""
        for b in range(B):
            for g in range(H_kv):
                g_gone = host[b][g].evict(before[b, g], keep, limit, first, last)
            gone[b] += 128 * g_gone
            assert cache.n_quant[b].item() == 128 * len(host[b][0].groups) and offset[b].item() == gone[b]

    evicted(mass.cpu().numpy())
    assert gone.tolist() == [(8 - keep) * 128, 0]

    # ---- generated tokens ----
    step_in = torch.zeros(B, 1, H_q + 2 * H_kv, 128, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    rows = [torch.zeros(B, h, 1, 128, dtype=torch.float16, device="cuda") for h in (H_q, H_kv, H_kv)]
    y, was = torch.zeros(B, H_q, 128, dtype=torch.float16, device="cuda"), torch.zeros_like(small)

    def step():
        cache.rotary(plan, step_in[:, :H_q], step_in[:, H_q:H_q + H_kv], step_in[:, H_q + H_kv:], first=offset, q_out=rows[0], k_out=rows[1], v_out=rows[2])
        cache.append(rows[1], rows[2])
        cache.decode_mass(rows[0].view(B, H_q, 128), small, out=y)
        was.copy_(small)
        cache.evict(small, keep, limit=limit, first=first, last=last, offset=offset)

    run = step
    if graph:
        saved = [t.clone() for t in (cache.groups, cache.k_res, cache.v_res, cache.n_quant, cache.n_res, small, offset)]
        step()  # (scratch at hand)
        for dst, src in zip((cache.groups, cache.k_res, cache.v_res, cache.n_quant, cache.n_res, small, offset), saved):
            dst.copy_(src)
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        run = captured.replay
    tokens = np.asarray(lengths)
    evictions = 0
    for i in range(steps):
        step_in.copy_(projected(1 + i, 1))
        before = small.cpu().numpy().astype(np.float64)
        run()
        torch.cuda.synchronize()
        r = [t.cpu().numpy() for t in rows]
        raw = step_in.double().cpu().numpy()
        look = i % 37 == 0 or i > steps - 3
        for b in range(B):
            if look:
                for got, want in ((r[0][b], raw[b, :H_q]), (r[1][b], raw[b, H_q:H_q + H_kv])):
                    z, off = bounded.rotated(want, [tokens[b] + i], freq, False, 1.1)
                    assert (np.abs(got.astype(np.float64) - z) <= off + bounded.rounding(z, "f16")).all(), (i, b)
            for g in range(H_kv):
                host[b][g].append(r[1][b, g, 0], r[2][b, g, 0])
        groups = [len(h[0].groups) for h in host]
        if look or any(n > limit for n in groups):
            accumulate(r[0], was, before)
            got = y.cpu().numpy()
            for b in range(B):
                for g in range(H_kv):
                    keys, values, _, _ = host[b][g].tokens()
                    if sliding and len(host[b][g].window) < 128:
                        tail = 128 - len(host[b][g].window)  # the newest 128 tokens: fp16 values, those of the newest group from its rows
                        n = len(keys)
                        values[n - 128:n - 128 + tail] = host[b][g].raw_values[-tail:]
                    for h in range(g * GQ, (g + 1) * GQ):
                        want, tol = ref.attend(r[0][b, h], keys, values, [len(keys) - 1])
                        ref.check_rows(got[b, h][None], want, tol, (i, b, h))
        evictions += sum(n > limit for n in groups)
        evicted(was.cpu().numpy())
    assert cache.status.item() == 0 and evictions >= 2
    assert (cache.n_quant + cache.n_res + offset).tolist() == [n + steps for n in lengths]
