"""Performance cases of the operators that read the packed cache beside the one-token decode: prompt attention, windowed decode, read-back.

Three kinds of pass, each one call on one layer's cache:

  "prompt"   KVLincCache.prompt_attention: T new tokens of every sequence attend to the cache and, causally, to their own rows
  "window"   KVLincCache.decode_windowed: one query of every sequence sees its newest `window` tokens and the first `sinks`
  "read"     KVLincCache.read: keys and values of T tokens of every sequence, dequantized

Fields of a case:
  B, Hq, Hkv     sequences, query heads, KV heads
  n              tokens of the longest sequence in the cache before the call; 0: an empty cache
  spread         the other sequences hold uniform in [n (1 - spread), n] tokens; 0: all alike
  T              rows of the call per sequence
  tspread        sequences take uniform in [T (1 - tspread), T] of these rows; 0: all of them (no count is given)
  bits           width of the codes
  corr           linear correction on
  sliding        the newest 128 tokens keep fp16 values
  window, sinks  newest tokens a query sees, first tokens that stay visible; window 0: everything
  dtype          of what is read back: "f16", "bf16" or "f32"
  rotated        values are read back in the rotated basis they are stored in
  tail           the newest T tokens are read back, not the first T

`run` computes a pass by plain torch operations in 32 bits from the packed buffers, or by the library's calls where `own` is set.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, kind, B, Hq, Hkv, n, T=1, spread=0.0, tspread=0.0, bits=2, corr=False, sliding=False, window=0, sinks=0, dtype="f16",
          rotated=False, tail=False):
    return {"name": name, "kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "n": n, "T": T, "spread": spread, "tspread": tspread, "bits": bits,
            "corr": corr, "sliding": sliding, "window": window, "sinks": sinks, "dtype": dtype, "rotated": rotated, "tail": tail}


def listed():
    return [
        # one chat prompt before anything is cached: a short causal attention
        _case("prompt_b1_700", "prompt", 1, 32, 8, 0, T=700),
        # a batch of prompts of unequal length, arriving together
        _case("prompt_b4_4k_ragged", "prompt", 4, 32, 8, 0, T=4096, tspread=0.6),
        # the next 8k tokens of a long document, over 24k cached ones with the correction: the largest call
        _case("prompt_b1_8k_over_24k", "prompt", 1, 32, 8, 24576, T=8192, corr=True),
        # a chunk of a prompt in a layer with a sliding window, 4-bit codes, seven query heads per KV head
        _case("prompt_chunk_window_gq7_4bit", "prompt", 2, 28, 4, 16384, T=1000, bits=4, window=4096, sinks=64),
        # drafted tokens of a batch, verified in one call
        _case("draft4_b16_8k", "prompt", 16, 32, 8, 8192, T=4, corr=True),
        # drafted tokens of one very long document
        _case("draft6_b1_128k", "prompt", 1, 32, 8, 131072, T=6, corr=True),
        # one user, a layer with a small window: the smallest call, latency bound
        _case("window1k_b1_8k", "window", 1, 32, 8, 8192, window=1024, sinks=4),
        # continuous batching: 64 users anywhere between 1k and 16k tokens
        _case("window4k_b64_ragged_16k", "window", 64, 32, 8, 16384, spread=0.9375, window=4096, sinks=128),
        # seven query heads per KV head, long contexts, a wide window, 4-bit codes
        _case("window8k_b32_32k_gq7_4bit", "window", 32, 28, 4, 32768, bits=4, window=8192, sinks=16),
        # a short chat moved to another worker
        _case("read_b1_300", "read", 1, 32, 8, 300, T=300),
        # a batch of 8k contexts read for reuse as plain fp16 keys and values
        _case("read_b16_8k", "read", 16, 32, 8, 8192, T=8192),
        # the newest tokens of a ragged batch with 4-bit codes, for a layer kept in bfloat16
        _case("read_tail_b32_4bit_bf16", "read", 32, 28, 4, 4100, T=1500, spread=0.5, bits=4, dtype="bf16", tail=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """Another case of the same ranges: sizes log-uniform and odd, at most the work of the largest listed case."""
    kind = rng.choice(["prompt", "prompt", "draft", "window", "window", "read"])
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (28, 4), (32, 32), (64, 8), (16, 8), (12, 2)])
    bits = 4 if rng.random() < 0.3 else 2
    B = _log(rng, 1, 64)
    sliding = rng.random() < 0.15
    spread = rng.choice([0.0, round(rng.uniform(0.05, 0.9), 2)]) if B > 1 else 0.0
    rows = 1_500_000 // (B * Hkv)                     # (sequence, KV head, token) rows of the cache
    if kind in ("prompt", "draft"):
        n = 0 if kind == "prompt" and rng.random() < 0.3 else _log(rng, 130, max(131, min(131072, rows)))
        if kind == "draft":
            T = rng.randint(1, 16)
        else:
            most = min(8192, 400_000 // (B * Hq), int(2e9 / (B * Hq * (n + 1))) + 16)
            T = _log(rng, 17, max(18, most))
        window = _log(rng, 16, 8192) if rng.random() < 0.35 else 0
        corr = window == 0 and n > 0 and rng.random() < 0.5
        c = _case("", "prompt", B, Hq, Hkv, n, T=T, spread=spread, tspread=rng.choice([0.0, round(rng.uniform(0.1, 0.9), 2)]), bits=bits,
                  corr=corr, sliding=sliding, window=window, sinks=rng.choice([0, 1, 4, rng.randint(1, 300)]) if window else 0)
    elif kind == "window":
        n = _log(rng, 1, max(2, min(131072, rows)))
        c = _case("", "window", B, Hq, Hkv, n, spread=spread, bits=bits, sliding=sliding, window=_log(rng, 1, 16384),
                  sinks=rng.choice([0, 1, 4, rng.randint(1, 300)]))
    else:
        n = _log(rng, 1, max(2, min(32768, rows)))
        c = _case("", "read", B, Hq, Hkv, n, T=_log(rng, 1, n), spread=spread, bits=bits, sliding=sliding, dtype=rng.choice(list(DTYPES)),
                  rotated=rng.random() < 0.3, tail=rng.random() < 0.5)
    del c["name"]
    return c


def _counts(most, spread, B, key):
    """B counts with the largest first, a function of the case alone (the work of a pass does not depend on the seed)."""
    if most == 0:
        return np.zeros(B, dtype=np.int64)
    out = np.random.default_rng([B, most, key]).integers(max(1, int(most * (1.0 - spread))), most + 1, size=B)
    out[0] = most
    return out.astype(np.int64)


def _lengths(case):
    """Cached tokens (quantized, in the window) and rows of the call of every sequence: whole groups of 128 leave a full window."""
    n = _counts(case["n"], case["spread"], case["B"], 7)
    nr = np.where(n > 0, (n - 1) % 128 + 1, 0)
    return n - nr, nr, _counts(case["T"], case["tspread"], case["B"], 11)


def _hadamard(dtype, device):
    h = torch.ones(1, 1, dtype=dtype, device=device)
    for _ in range(7):
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h * 128 ** -0.5


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _quantized(x, dim, bits):
    """Codes, scale and zero-point of groups of 128 along `dim`: zero-point = minimum, scale = range / levels in binary16, nearest code."""
    levels = 2 ** bits - 1
    zero = x.amin(dim, keepdim=True)
    scale = ((x.amax(dim, keepdim=True).float() - zero.float()) / levels).half()
    codes = ((x.float() - zero.float()) / scale.float()).round_().clamp_(0, levels).to(torch.uint8)
    return codes, scale, zero


def _logical(case, seed):
    """What the cache stands for, and the call's inputs: codes [B, Hkv, G, token, channel] with their scales, window rows, new rows."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, dtype=torch.float16, device=dev, generator=gen)
    B, Hq, Hkv, T = case["B"], case["Hq"], case["Hkv"], case["T"]
    nq, nr, rows = _lengths(case)
    G = max(1, int(nq.max()) // 128)
    # keys N(0, 1) with 4 channels per KV head 8 times as large; values N(0, 1), which the rotation leaves as they are
    gain = torch.ones(Hkv, 128, dtype=torch.float16, device=dev)
    gain.scatter_(1, torch.rand(Hkv, 128, device=dev, generator=gen).argsort(1)[:, :4], 8.0)
    d = {"nq": nq, "nr": nr, "rows": rows, "G": G}
    x = normal(B, Hkv, G, 128, 128).mul_(gain[:, None, None, :])
    d["kc"], d["ks"], d["kz"] = _quantized(x, 3, case["bits"])
    x = normal(B, Hkv, G, 128, 128)
    d["vc"], d["vs"], d["vz"] = _quantized(x, 4, case["bits"])
    del x
    d["k_win"] = normal(B, Hkv, 128, 128).mul_(gain[:, None, :])
    d["v_win"] = normal(B, Hkv, 128, 128)
    if case["kind"] != "read":
        d["q"] = normal(B, Hq, T, 128) if case["kind"] == "prompt" else normal(B, Hq, 128)
    if case["kind"] == "prompt":
        d["k_new"] = normal(B, Hkv, T, 128).mul_(gain[:, None, :])
        d["v_new"] = normal(B, Hkv, T, 128)
    if case["corr"]:
        # states of n quantized tokens: features near 1 / 128 a token, summed with the values' signs
        n = torch.from_numpy(nq.astype(np.float32)).to(dev)[:, None, None]
        d["Wq"] = normal(Hq, 2, 128, 128).mul_(128 ** -0.5)
        d["Wk"] = normal(Hkv, 2, 128, 128).mul_(128 ** -0.5)
        d["P"] = n / 128 * (1 + 0.1 * torch.randn(B, Hkv, 256, device=dev, generator=gen)).clamp_min_(0.1)
        d["S"] = (n[..., None].sqrt() / 128 * torch.randn(B, Hkv, 256, 128, device=dev, generator=gen)).half()
    if case["kind"] == "read":
        total = nq + nr
        d["first"] = np.maximum(total - T, 0) if case["tail"] else np.zeros(B, dtype=np.int64)
    return d


def _value_order(dev):
    """Token of position k of a row of a value tile."""
    k = torch.arange(128, device=dev)
    return 16 * (k % 8) + 4 * ((k // 16) % 4) + 2 * (k // 64) + (k // 8) % 2


def _packed(codes):
    """2-bit codes [..., 128 rows, 128 positions] to words [..., 1024]."""
    c = codes.view(*codes.shape[:-2], 4, 2, 16, 4, 2, 2, 8).int()                # n / 2, n % 2, j, g, w, parity, i
    pair = (1 - (c >> 1)) << 3 | (1 ^ (c & 1) ^ (c >> 1)) << 1                   # (hi, lo) in bits 3 and 1 of a nibble
    words = ((pair >> torch.arange(2, device=c.device)[:, None].int()) << (4 * torch.arange(8, device=c.device)).int()).sum((-1, -2)).int()
    lead = list(range(words.dim() - 5))
    k = len(lead)
    return words.permute(*lead, k, k + 3, k + 2, k + 1, k + 4).reshape(*words.shape[:k], 1024)


def _planes(codes, bits):
    return _packed(codes) if bits == 2 else torch.cat((_packed(codes >> 2), _packed(codes & 3)), -1)


def _device_counts(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).to(dev)


def prepare(case, seed):
    d = _logical(case, seed)
    dev = d["k_win"].device
    B, Hkv, T, G = case["B"], case["Hkv"], case["T"], d["G"]
    pairs = lambda lo, hi: torch.stack((lo, hi), -1).contiguous().view(torch.int32)[..., 0]
    scales = lambda t: t[..., 0, :].contiguous().view(torch.int32)              # [.., 1, 128] halves to 64 words
    sz = pairs(d["vs"][..., 0], d["vz"][..., 0])                                 # word 8 j + n is token 16 n + j
    sz = sz.view(B, Hkv, G, 8, 16).transpose(-1, -2).reshape(B, Hkv, G, 128)
    values = d["vc"].transpose(-1, -2)[..., _value_order(dev)]
    groups = torch.cat((_planes(d["kc"], case["bits"]), _planes(values, case["bits"]), scales(d["ks"]), scales(d["kz"]), sz), -1).contiguous()
    state = {"case": case, "groups": groups, "k_res": d["k_win"].contiguous(),
             "v_res": d["v_win"].view(B, Hkv, 32, 4, 128).transpose(-1, -2).contiguous(),
             "n_quant": _device_counts(d["nq"], dev), "n_res": _device_counts(d["nr"], dev), "longest": max(1, int((d["nq"] + d["nr"]).max()))}
    for k in ("q", "k_new", "v_new", "Wq", "Wk", "P"):
        state[k] = d.get(k)
    if case["corr"]:  # tile (64-feature block, channel half, 4-feature step) holds [channel % 64][feature % 4]
        state["S16"] = d["S"].view(B, Hkv, 4, 16, 4, 2, 64).permute(0, 1, 2, 5, 3, 6, 4).reshape(B, Hkv, 128, 64, 4).contiguous()
    if case["kind"] == "prompt":
        state["n_new"] = _device_counts(d["rows"], dev) if case["tspread"] > 0 else None
    if case["kind"] == "read":
        state["first"] = _device_counts(d["first"], dev) if case["tail"] else None
        state["k_out"] = torch.zeros(B, Hkv, T, 128, dtype=DTYPES[case["dtype"]], device=dev)
        state["v_out"] = torch.zeros_like(state["k_out"])
    else:
        state["out"] = torch.zeros_like(state["q"])
    if own:
        state["cache"] = _cache(state)
    return state


def _cache(state):
    import paper_2510_05373_amd as kv
    case = state["case"]
    room = 128 * state["groups"].shape[2] + (case["T"] if case["kind"] == "prompt" else 0)
    cache = kv.KVLincCache(case["B"], case["Hq"], case["Hkv"], room, Wq=state["Wq"], Wk=state["Wk"], bits=case["bits"],
                           flags=kv.KVLINC_FLAG_SLIDING_VALUES if case["sliding"] else 0)
    cache.groups[:, :, :state["groups"].shape[2]].copy_(state["groups"])
    state["groups"] = None
    cache.k_res.copy_(state["k_res"])
    cache.v_res.copy_(state["v_res"])
    cache.n_quant.copy_(state["n_quant"])
    cache.n_res.copy_(state["n_res"])
    if case["corr"]:
        cache.S16.copy_(state["S16"])
        cache.P.copy_(state["P"])
    return cache


def run(state):
    case = state["case"]
    if own:
        cache = state["cache"]
        if case["kind"] == "prompt":
            return [cache.prompt_attention(state["q"], state["k_new"], state["v_new"], n_new=state["n_new"], window=case["window"],
                                           sinks=case["sinks"], out=state["out"], max_context=state["longest"])]
        if case["kind"] == "window":
            return [cache.decode_windowed(state["q"], case["window"], sinks=case["sinks"], out=state["out"], max_context=state["longest"])]
        return list(cache.read(first=state["first"], T=case["T"], dtype=DTYPES[case["dtype"]], rotated=case["rotated"], k_out=state["k_out"],
                               v_out=state["v_out"]))
    return _read(state) if case["kind"] == "read" else _attention(state)


# ---- plain form ---------------------------------------------------------------------------------------------------------

def _unpacked(words):
    """Words [..., 1024] to 2-bit codes [..., 128 rows, 128 positions]."""
    dev = words.device
    lead, k = words.shape[:-1], words.dim() - 1
    w = words.reshape(*lead, 4, 4, 16, 2, 2)                                     # n / 2, g, j, n % 2, w
    w = w.permute(*range(k), k, k + 3, k + 2, k + 1, k + 4).reshape(*lead, 128, 8, 1, 1)
    at = 4 * torch.arange(8, device=dev) - torch.arange(2, device=dev)[:, None]  # parity, i
    code = torch.tensor([2, 3, 1, 0], dtype=torch.uint8, device=dev)             # of the pair hi lo
    return code[((w >> (at + 3).int()) & 1) << 1 | ((w >> (at + 1).int()) & 1)].reshape(*lead, 128, 128)


def _tile(words, bits):
    return _unpacked(words).float() if bits == 2 else 4.0 * _unpacked(words[..., :1024]).float() + _unpacked(words[..., 1024:]).float()


def _halves(words):
    return words.contiguous().view(torch.float16).float()


def _dequantized(records, bits):
    """Records [..., words] to keys and rotated values [..., 128 tokens, 128 channels]."""
    t = 512 * bits
    key = _tile(records[..., :t], bits) * _halves(records[..., 2 * t:2 * t + 64])[..., None, :] + _halves(records[..., 2 * t + 64:2 * t + 128])[..., None, :]
    order = torch.argsort(_value_order(records.device))
    value = _tile(records[..., t:2 * t], bits).transpose(-1, -2)[..., order, :]
    sz = _halves(records[..., 2 * t + 128:]).reshape(*records.shape[:-1], 16, 8, 2).transpose(-2, -3).reshape(*records.shape[:-1], 128, 2)
    return key, value * sz[..., :1] + sz[..., 1:]


def _window_values(state):
    v = state["v_res"].float()
    return v.transpose(-1, -2).reshape(*v.shape[:2], 128, 128)


def _context(state, index):
    """Keys and rotated values of the groups `index` [B, k] and of the window, [B, Hkv, tokens, 128], and the tokens' positions [B, tokens]
    with -1 where there is none."""
    case = state["case"]
    B, Hkv = case["B"], case["Hkv"]
    nq, nr = state["n_quant"].long()[:, None], state["n_res"].long()[:, None]
    dev = nq.device
    key, value = _dequantized(state["groups"][torch.arange(B, device=dev)[:, None], :, index].transpose(1, 2), case["bits"])
    slot = torch.arange(128, device=dev)
    at = index[..., None] * 128 + slot                                           # [B, k, 128]
    v_win = _window_values(state)
    if case["sliding"]:
        kept = (at >= nq[..., None] + nr[..., None] - 128)[:, None, :, :, None]
        value = torch.where(kept, v_win[:, :, None], value)
    at = torch.where(at < nq[..., None], at, -1).flatten(1)
    at_win = torch.where(slot < nr, nq + slot, -1)
    return (torch.cat((key.flatten(2, 3), state["k_res"].float()), 2), torch.cat((value.flatten(2, 3), v_win), 2), torch.cat((at, at_win), 1))


def _attention(state):
    case = state["case"]
    B, Hq, Hkv, T, window, sinks = case["B"], case["Hq"], case["Hkv"], case["T"], case["window"], case["sinks"]
    prompt = case["kind"] == "prompt"
    total = (state["n_quant"] + state["n_res"]).long()[:, None]
    dev = total.device
    G = state["groups"].shape[2]
    p = total + torch.arange(T, device=dev) if prompt else total - 1             # positions of the queries [B, T]
    if window and window + T < state["longest"]:
        # the groups with first tokens, then those of the newest tokens; a token that is in both counts in the second
        low = (p[:, :1] - window + 1).clamp_min(0)
        n_first, n_last = -(-sinks // 128), -(-(window + T) // 128) + 1
        first = torch.arange(n_first, device=dev).expand(B, -1)
        last = low // 128 + torch.arange(n_last, device=dev)
        key, value, at = _context(state, torch.cat((first, last), 1).clamp_max(G - 1))
        n_first = 128 * n_first
        at[:, :n_first] = torch.where(at[:, :n_first] < low // 128 * 128, at[:, :n_first], -1)
        at[:, n_first:-128] = torch.where((last[..., None] < G).expand(-1, -1, 128).flatten(1), at[:, n_first:-128], -1)
    else:
        key, value, at = _context(state, torch.arange(G, device=dev).expand(B, -1))
    value = value @ _hadamard(torch.float32, dev)
    if prompt:
        key, value = torch.cat((key, state["k_new"].float()), 2), torch.cat((value, state["v_new"].float()), 2)
        at = torch.cat((at, p), 1)
    q = state["q"].float().view(B, Hkv, -1, 128)                                 # rows = (head of the KV head, token)
    s = (q @ key.transpose(-1, -2)).mul_(128 ** -0.5).view(B, Hkv, Hq // Hkv, T, -1)
    d = p[:, :, None] - at[:, None, :]
    hidden = (d < 0) | (at[:, None, :] < 0)
    if window:
        hidden |= (d >= window) & (at[:, None, :] >= sinks)
    s.masked_fill_(hidden[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    if case["corr"]:
        m = m.clamp_min(0.0)
    m = torch.where(m == -math.inf, 0.0, m)
    s.sub_(m).exp_()
    den = s.sum(-1, keepdim=True)
    num = (s.view(B, Hkv, -1, s.shape[-1]) @ value).view(B, Hkv, Hq // Hkv, T, 128)
    if case["corr"]:
        logits = state["q"].float()[:, :, None] @ state["Wq"].float()           # [B, Hq, 2, T, 128]
        e = (logits - logits.amax(-1, keepdim=True)).exp()
        phi = (e / e.sum(-1, keepdim=True)).transpose(2, 3).reshape(B, Hkv, -1, 256)
        S = state["S16"].float().view(B, Hkv, 4, 2, 16, 64, 4).permute(0, 1, 2, 4, 6, 3, 5).reshape(B, Hkv, 256, 128)
        C = (phi @ S @ _hadamard(torch.float32, dev)).view(num.shape)
        w = (-m).exp()
        num = num + w * C
        den = den + w * (phi @ state["P"][..., None]).view(den.shape)
    out = (num / den).view(B, Hq, T, 128)
    if not prompt:
        return [torch.where(total[..., None] > 0, out[:, :, 0], 0.0).half()]
    if state["n_new"] is not None:
        out = torch.where((torch.arange(T, device=dev) < state["n_new"][:, None])[:, None, :, None], out, 0.0)
    return [out.half()]


def _read(state):
    case = state["case"]
    B, Hkv, T = case["B"], case["Hkv"], case["T"]
    dev = state["n_quant"].device
    G = state["groups"].shape[2]
    key, value, at = _context(state, torch.arange(G, device=dev).expand(B, -1))
    if not case["rotated"]:
        value = value @ _hadamard(torch.float32, dev)
    nq, total = state["n_quant"].long()[:, None], (state["n_quant"] + state["n_res"]).long()[:, None]
    t = torch.arange(T, device=dev).expand(B, -1)
    if state["first"] is not None:
        t = t + state["first"].long()[:, None]
    there = (t < total)[:, None, :, None]
    row = torch.where(t < nq, t, 128 * G + t - nq).clamp_max(at.shape[1] - 1)    # the window's rows follow the groups'
    pick = lambda x: torch.where(there, x[torch.arange(B, device=dev)[:, None], :, row].transpose(1, 2), 0.0).to(DTYPES[case["dtype"]])
    return [pick(key), pick(value)]


# ---- the same in 64 bits, from what the codes stand for --------------------------------------------------------------------

def _visible(case, p, low, high):
    """Tokens low .. high - 1 that a query at position p [T] sees: [T, high - low]."""
    j = torch.arange(low, high, device=p.device)
    seen = j <= p[:, None]
    if case["window"]:
        seen &= (j > p[:, None] - case["window"]) | (j < case["sinks"])
    return seen


def exact(case, seed):
    d = _logical(case, seed)
    dev = d["k_win"].device
    B, Hq, Hkv, T = case["B"], case["Hq"], case["Hkv"], case["T"]
    if case["kind"] == "read" and 2 * B * Hkv * T * 128 > 600e6:
        return None
    gq = Hq // Hkv
    H = _hadamard(torch.float64, dev)
    if case["kind"] == "read":
        result = [torch.zeros(B, Hkv, T, 128, dtype=torch.float64, device=dev) for _ in range(2)]
    else:
        result = [torch.zeros(d["q"].shape, dtype=torch.float64, device=dev)]
    for b in range(B):
        nq, nr = int(d["nq"][b]), int(d["nr"][b])
        n, G = nq + nr, nq // 128
        rows = int(d["rows"][b]) if case["kind"] == "prompt" else 1
        for g in range(Hkv):
            key = d["kc"][b, g, :G].double() * d["ks"][b, g, :G].double() + d["kz"][b, g, :G].double()
            val = d["vc"][b, g, :G].double() * d["vs"][b, g, :G].double() + d["vz"][b, g, :G].double()
            key = torch.cat((key.reshape(-1, 128), d["k_win"][b, g, :nr].double()))
            val = torch.cat((val.reshape(-1, 128), d["v_win"][b, g, :nr].double()))
            if case["sliding"] and G and nr < 128:
                val[n - 128:nq] = d["v_win"][b, g, nr:].double()
            if case["kind"] == "read":
                a = int(d["first"][b])
                e = min(n, a + T)
                if e > a:
                    result[0][b, g, :e - a] = key[a:e]
                    result[1][b, g, :e - a] = val[a:e] if case["rotated"] else val[a:e] @ H
                continue
            val = val @ H
            if case["kind"] == "prompt":
                key = torch.cat((key, d["k_new"][b, g, :rows].double()))
                val = torch.cat((val, d["v_new"][b, g, :rows].double()))
            for h in range(g * gq, (g + 1) * gq):
                q = d["q"][b, h].double().view(-1, 128)[:rows]
                for i in range(0, rows, 2048):
                    x = q[i:i + 2048]
                    p = (n if case["kind"] == "prompt" else n - 1) + i + torch.arange(x.shape[0], device=dev)
                    if n == 0 and case["kind"] == "window":
                        continue
                    w = (x @ key.T / math.sqrt(128.0)).masked_fill_(~_visible(case, p, 0, key.shape[0]), -math.inf)
                    shift = w.amax(1, keepdim=True)
                    w = (w - shift).exp_()
                    num, den = w @ val, w.sum(1, keepdim=True)
                    if case["corr"]:
                        phi = torch.cat([(x @ d["Wq"][h, k].double()).softmax(1) for k in range(2)], 1)
                        num = num + (-shift).exp() * (phi @ d["S"][b, g].double() @ H)
                        den = den + (-shift).exp() * (phi @ d["P"][b, g].double())[:, None]
                    y = num / den
                    if case["kind"] == "prompt":
                        result[0][b, h, i:i + x.shape[0]] = y
                    else:
                        result[0][b, h] = y[0]
    return result


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------

def _seen(case, n, rows):
    """(query, key) pairs of one head, and cached tokens that some query sees: (pairs, quantized part, window part) of one sequence."""
    prompt = case["kind"] == "prompt"
    p = n + np.arange(rows, dtype=np.int64) if prompt else np.array([n - 1], dtype=np.int64)
    if n == 0 and not prompt:
        return 0, 0, 0
    nr = (n - 1) % 128 + 1 if n else 0
    nq = n - nr
    w, s = case["window"], case["sinks"]
    pairs = int((p + 1).sum()) if not w else int((np.minimum(p + 1, w) + np.minimum(s, np.maximum(p + 1 - w, 0))).sum())
    low = max(0, int(p[0]) - w + 1) if w else 0
    quant = nq if low == 0 else min(s, low, nq) + max(0, nq - low)
    return pairs, quant, (nr if low <= nq else max(0, n - low))


def work(case):
    B, Hq, Hkv = case["B"], case["Hq"], case["Hkv"]
    nq, nr, rows = _lengths(case)
    token = 32 * case["bits"] + 8                    # bytes of a quantized token of one KV head
    byts = flops = 0.0
    size = {"f16": 2, "bf16": 2, "f32": 4}[case["dtype"]]
    for b in range(B):
        n = int(nq[b] + nr[b])
        if case["kind"] == "read":
            a = max(0, n - case["T"]) if case["tail"] else 0
            e = min(n, a + case["T"])
            quant = max(0, min(e, int(nq[b])) - a)
            byts += Hkv * (quant * token + (e - a - quant) * 512 + (e - a) * 256 * size)
            flops += Hkv * (e - a) * 128 * (4 if case["rotated"] else 11)
            continue
        r = int(rows[b]) if case["kind"] == "prompt" else 1
        pairs, quant, win = _seen(case, n, r)
        byts += Hkv * (quant * token + win * 512) + Hq * r * 512 + (Hkv * r * 512 if case["kind"] == "prompt" else 0)
        flops += Hq * pairs * 512.0
        if case["corr"]:
            byts += Hkv * (65536 + 1024)
            flops += Hq * r * 4.0 * 128 * 256
    if case["corr"]:
        byts += Hq * 65536
    return {"bytes": byts, "flops": flops}
