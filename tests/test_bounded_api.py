"""Host side of kvlinc_bounded.h: exported names, what is refused before any launch, workspace sizes, and the checks of KVLincCache.
No compute call is made here."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2510_05373_amd as kv
from paper_2510_05373_amd import binding as kb
from tests.test_library_abi import fake_struct

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "kvlinc_bounded.h")
NONE = dict(S=0, S16=0, P=0, Wq=0, Wk=0)


def plain(**over):
    return fake_struct(**{**NONE, **over})


def p(a):
    return None if a is None else ctypes.c_void_p(a)


def test_header_functions_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(kvlinc_[a-z_]+)\s*\(", text)))
    assert names == ["kvlinc_attention_mass", "kvlinc_attention_mass_workspace_bytes", "kvlinc_cache_evict", "kvlinc_cache_evict_workspace_bytes",
                     "kvlinc_decode_attention_mass", "kvlinc_decode_mass_workspace_bytes", "kvlinc_rotary"]
    lib = ctypes.CDLL(kb.lib_path)
    for n in names:
        assert hasattr(lib, n) and callable(getattr(kv, n))


@pytest.mark.parametrize("name, mirror", [("kvlinc_rotation", kb.RotationStruct), ("kvlinc_rows", kb.RowsStruct)])
def test_struct_mirrors_match_the_header(name, mirror):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = text[text.index("typedef struct %s {" % name):text.index("} %s;" % name)].split("{", 1)[1]
    fields = [re.findall(r"(\w+)$", part.strip())[0] for line in body.split(";") if line.strip() for part in line.split(",")]
    assert fields == [n.rstrip("_") for n, _ in mirror._fields_]


# ---- positions -------------------------------------------------------------------------------------------------------------------

def rows(at=0x100000, out=0x200000, strides=(8 * 4 * 128, 4 * 128, 128)):
    return kb.RowsStruct(at, out, *strides)


def rotary(c=None, rot=None, q="rows", k=None, v=None, T=4, n_new=None, first=None, depth=None, counted=1, din=0, dout=0, **over):
    rot = rot or kb.RotationStruct(**{**dict(channels=128, interleaved=0, magnitude=1.0, freq=0x10000), **over})
    return kb.lib.kvlinc_rotary(ctypes.byref(c or plain()), rot, rows() if q == "rows" else q, k, v, T, p(n_new), p(first), p(depth), counted, din, dout, None)


@pytest.mark.parametrize("over", [
    dict(channels=0), dict(channels=-2), dict(channels=63), dict(channels=130), dict(interleaved=2), dict(interleaved=-1), dict(magnitude=math.inf),
    dict(magnitude=math.nan), dict(freq=0), dict(freq=0x10008), dict(q=None), dict(q=rows(at=None)), dict(q=rows(at=0x100008)), dict(q=rows(out=None)),
    dict(q=rows(out=0x200004)), dict(q=rows(strides=(-128, 128, 128))), dict(q=rows(strides=(4096, 512, 132))), dict(q=rows(strides=(4096, 516, 128))),
    dict(q=rows(strides=((1 << 48) + 8, 512, 128))), dict(T=0), dict(T=-1), dict(T=(1 << 24) + 1), dict(T=1 << 25), dict(n_new=0x20002), dict(first=0x20001),
    dict(depth=0x20003), dict(counted=2), dict(counted=-1), dict(din=3), dict(din=-1), dict(dout=3), dict(dout=-1)])
def test_rotary_refuses(over):
    assert rotary(**over) == kb.KVLINC_EINVAL


def test_rotary_refuses_without_descriptors():
    assert rotary(fake_struct(d=64)) == kb.KVLINC_EINVAL
    assert kb.lib.kvlinc_rotary(None, kb.RotationStruct(128, 0, 1.0, 0x10000), rows(), None, None, 1, None, None, None, 1, 0, 0, None) == kb.KVLINC_EINVAL
    assert kb.lib.kvlinc_rotary(ctypes.byref(plain()), None, rows(), None, None, 1, None, None, None, 1, 0, 0, None) == kb.KVLINC_EINVAL
    assert rotary(plain(B=1 << 20), T=64) == kb.KVLINC_EINVAL  # 2^26 tokens


def test_rotary_refuses_shared_memory():
    c = plain()  # B 2, H_q 8, H_kv 2; T 4: queries 16384 bytes, keys 4096
    at, q_bytes = 0x100000, 2 * 8 * 4 * 256
    whole = (8 * 4 * 128, 4 * 128, 128)
    kv_whole = (2 * 4 * 128, 4 * 128, 128)
    bad = [dict(q=rows(at, at + 16, whole)), dict(q=rows(at, at + q_bytes - 16, whole)), dict(q=rows(at, at - q_bytes + 16, whole)),
           dict(q=rows(at, at, whole), dout=2),                       # in place, of another type
           dict(q=rows(at, at, (8 * 128 * 4, 128, 8 * 128))),         # in place, of another layout
           dict(q=rows(at, 0x800000, whole), k=rows(0x400000, 0x800000 + q_bytes - 16, kv_whole)),  # two outputs
           dict(q=rows(at, 0x800000, whole), k=rows(0x800000 + 16, 0x900000, kv_whole)),            # one's output, the other's input
           dict(q=rows(at, at + 256, (12 * 4 * 128, 128, 12 * 128)))]  # between the rows of a projection's output
    for over in bad:
        assert rotary(c, **over) == kb.KVLINC_EINVAL, over


def test_frequencies():
    f = kv.rotary_frequencies(8, base=10000.0)
    assert f == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-14)
    assert kv.rotary_frequencies(8, scaling="linear", factor=4.0) == pytest.approx([x / 4 for x in f], rel=1e-14)
    based = kv.rotary_frequencies(8, scaling="base", factor=4.0)
    assert based[0] == 1.0 and based[-1] == pytest.approx(f[-1] / 4, rel=1e-12) and f[1] / 4 < based[1] < f[1]
    # 628.3 tokens: the pairs turn 100, 10, 1 and 0.1 times in them
    parts = kv.rotary_frequencies(8, scaling="parts", factor=4.0, original=200 * math.pi, low=1.0, high=19.0)
    assert parts[0] == 1.0 and parts[1] == pytest.approx(0.5 * f[1] + 0.5 * f[1] / 4, rel=1e-12) and parts[2:] == pytest.approx([x / 4 for x in f[2:]], rel=1e-12)
    assert kv.rotary_frequencies(2, scaling="base", factor=2.0) == [1.0]
    for bad in (dict(channels=7), dict(channels=0), dict(channels=130), dict(base=0.0), dict(factor=0.0), dict(scaling="other"), dict(scaling="parts", factor=2.0),
                dict(scaling="parts", factor=2.0, original=10, low=3.0, high=3.0), dict(base=math.nan)):
        with pytest.raises(kv.KVLincError):
            kv.rotary_frequencies(**bad)


@pytest.mark.parametrize("freq, over", [([], {}), ([1.0] * 65, {}), ([[1.0, 2.0]], {}), ([1.0], dict(magnitude=math.nan))])
def test_a_rotation_checks_its_numbers(freq, over):
    with pytest.raises(kv.KVLincError):
        kv.KVLincRotary(freq, device="cpu", **over)


def test_the_rotation_back():
    a = kv.KVLincRotary([1.0, 0.5], interleaved=True, magnitude=2.0, device="cpu")
    b = a.inverse()
    assert b.freq.tolist() == [-1.0, -0.5] and b.magnitude == 0.5 and b.interleaved and b.channels == 4
    with pytest.raises(kv.KVLincError):
        kv.KVLincRotary([1.0], magnitude=0.0, device="cpu").inverse()


# ---- accumulated attention weight ------------------------------------------------------------------------------------------------

def decode(c, q=0x200000, out=0x300000, mass=0x400000, decay=1.0, mass_out=0x500000, ws=0x800000, size=1 << 40, bound=0):
    return kb.lib.kvlinc_decode_attention_mass(ctypes.byref(c), p(q), p(out), p(mass), decay, p(mass_out), p(ws), size, bound, None)


def of_rows(c, q=0x200000, n=None, T=4, mass=0x400000, decay=1.0, mass_out=0x500000, ws=0x800000, size=1 << 40, bound=0):
    return kb.lib.kvlinc_attention_mass(ctypes.byref(c), p(q), p(n), T, p(mass), decay, p(mass_out), p(ws), size, bound, None)


MASS = [dict(q=None), dict(q=0x200008), dict(mass=0x400002), dict(mass_out=None), dict(mass_out=0x500001), dict(decay=-0.1), dict(decay=1.5), dict(decay=math.nan),
        dict(mass=0x500004), dict(mass_out=0x200010)]


@pytest.mark.parametrize("over", MASS + [dict(out=None), dict(out=0x300004), dict(out=0x200010), dict(mass_out=0x300010), dict(out=0x400010)])
def test_decode_with_mass_refuses(over):
    assert decode(plain(), **over) == kb.KVLINC_EINVAL


@pytest.mark.parametrize("over", MASS + [dict(n=0x20002), dict(T=0), dict(T=-1), dict(T=(1 << 20) + 1)])
def test_mass_of_rows_refuses(over):
    assert of_rows(plain(), **over) == kb.KVLINC_EINVAL


def test_adapters_are_refused():
    full = fake_struct()
    assert decode(full) == of_rows(full) == kb.KVLINC_EINVAL
    assert kb.kvlinc_decode_mass_workspace_bytes(full) == kb.kvlinc_attention_mass_workspace_bytes(full, 4) == kb.kvlinc_cache_evict_workspace_bytes(full) == 0
    assert evict(full, full, to_at=None) == evict(plain(), full) == kb.KVLINC_EINVAL


@pytest.mark.parametrize("shape", [dict(d=64), dict(B=1 << 24, H_q=1, H_kv=1), dict(B=1, H_q=1, H_kv=1, max_groups=1 << 24), dict(B=1 << 12, H_kv=2, max_groups=1 << 14)])
def test_shapes_beyond_the_limits_are_refused(shape):
    c = plain(**shape)
    assert decode(c) == of_rows(c) == kb.KVLINC_EINVAL
    assert kb.kvlinc_decode_mass_workspace_bytes(c) == kb.kvlinc_attention_mass_workspace_bytes(c, 4) == kb.kvlinc_cache_evict_workspace_bytes(c) == 0


def test_more_rows_than_a_grid_holds_are_refused():
    c = plain(B=256, H_q=32, H_kv=32, max_groups=64)
    assert of_rows(c, T=1 << 15) == kb.KVLINC_EINVAL and kb.kvlinc_attention_mass_workspace_bytes(c, 1 << 15) == 0
    assert kb.kvlinc_attention_mass_workspace_bytes(c, 64) > 0


def test_workspaces():
    c = plain(max_groups=64)
    need = kb.kvlinc_decode_mass_workspace_bytes(c)
    assert need >= 2 * 2 * 68 * 64
    for over in (dict(ws=None), dict(ws=0x800008), dict(size=need - 1)):
        assert decode(c, **over) == kb.KVLINC_EWORKSPACE
    assert decode(c, out=0x200000, mass_out=0x400000, size=0) == kb.KVLINC_EWORKSPACE  # (both in place: allowed)
    # a bound makes it no smaller than what any sequence of the cache needs
    assert kb.kvlinc_decode_mass_workspace_bytes(c, 1) >= 2 * 2 * 68 * 64
    need = kb.kvlinc_attention_mass_workspace_bytes(c, 4)
    assert need == 4 * 2 * 2 * 16 * (65 + 1)  # rows of a KV head: 16; a number for each of them and slot, and one more
    for over in (dict(ws=None), dict(ws=0x800008), dict(size=need - 1)):
        assert of_rows(c, **over) == kb.KVLINC_EWORKSPACE
    assert kb.kvlinc_attention_mass_workspace_bytes(c, 4, 300) == 4 * 2 * 2 * 16 * (4 + 1)
    assert {kb.kvlinc_attention_mass_workspace_bytes(c, 4, n) for n in (0, -7, 1 << 30)} == {need}


# ---- eviction --------------------------------------------------------------------------------------------------------------------

FAR = dict(groups=0x40000000, k_res=0x50000000, v_res=0x52000000, n_quant=0x54000000, n_res=0x55000000)
NEAR = dict(groups=0x10000000, k_res=0x20000000, v_res=0x22000000, n_quant=0x24000000, n_res=0x25000000)


def evict(a=None, b=None, to_at="far", mass=0x60000000, mass_out=0x61000000, keep=4, limit=4, first=1, last=1, offset=None, offset_out=None, kept=None,
          ws=0x70000000, size=1 << 40, **shape):
    a = a if a is not None else plain(**NEAR)
    b = b if b is not None else plain(**{**(FAR if to_at == "far" else NEAR), **shape})
    return kb.lib.kvlinc_cache_evict(ctypes.byref(a), ctypes.byref(b), p(mass), p(mass_out), keep, limit, first, last, p(offset), p(offset_out), p(kept), p(ws), size, None)


@pytest.mark.parametrize("over", [
    dict(keep=0), dict(keep=-1), dict(limit=3), dict(first=-1), dict(last=0), dict(last=-1), dict(first=4), dict(first=2, last=3), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
    dict(mass=None), dict(mass=0x60000002), dict(mass_out=None), dict(mass_out=0x61000001), dict(offset=0x20001), dict(offset_out=0x20002), dict(kept=0x20003),
    dict(B=1), dict(H_q=4), dict(H_kv=4), dict(R=64), dict(bits=4), dict(flags=kb.KVLINC_FLAG_SLIDING_VALUES), dict(max_groups=3),
    dict(mass_out=0x60000010), dict(mass_out=0x60000000, max_groups=7), dict(offset=0x60000000, offset_out=0x60000004), dict(kept=0x61000000),
    dict(kept=0x40000000), dict(mass_out=0x40000000), dict(mass_out=0x10000000), dict(offset_out=0x24000000), dict(offset_out=0x60000000)])
def test_evict_refuses(over):
    assert evict(**over) == kb.KVLINC_EINVAL


def test_evict_refuses_half_of_a_cache_in_place():
    for name in FAR:
        assert evict(b=plain(**{**FAR, name: NEAR[name]})) == kb.KVLINC_EINVAL, name
        assert evict(b=plain(**{**NEAR, name: FAR[name]})) == kb.KVLINC_EINVAL, name
    assert evict(b=plain(**{**NEAR, "max_groups": 9})) == kb.KVLINC_EINVAL
    assert evict(to_at="near", size=0) == kb.KVLINC_EWORKSPACE  # (all of it: allowed)
    assert evict(to_at="near", mass_out=0x60000000, offset=0x20000, offset_out=0x20000, size=0) == kb.KVLINC_EWORKSPACE


def test_evict_needs_its_workspace():
    need = kb.kvlinc_cache_evict_workspace_bytes(plain())
    assert need > 0
    for over in (dict(ws=None), dict(ws=0x70000008), dict(size=need - 1)):
        assert evict(**over) == kb.KVLINC_EWORKSPACE
    # room for as many groups as the first cache has will do, whatever the limit
    assert evict(limit=1000, size=0) == kb.KVLINC_EWORKSPACE


# ---- KVLincCache: what it looks at before it hands out an address ----------------------------------------------------------------

@pytest.fixture(scope="module")
def cache():
    return kv.KVLincCache(2, 8, 2, 256, device="cpu")


@pytest.fixture(scope="module")
def plan():
    return kv.KVLincRotary(kv.rotary_frequencies(64), device="cpu")


def half(*s):
    return torch.zeros(*s, dtype=torch.float16)


def ints(*s):
    return torch.zeros(*s, dtype=torch.int32)


@pytest.mark.parametrize("over", [
    dict(q=None), dict(q=half(2, 8, 128)), dict(q=half(2, 4, 3, 128)), dict(q=half(2, 8, 3, 64)), dict(q=half(2, 8, 3, 128).double()), dict(q=half(2, 8, 3, 256)[..., ::2]),
    dict(q=half(2, 8, 0, 128)), dict(k=half(2, 8, 3, 128)), dict(k=half(2, 2, 4, 128)), dict(k=half(2, 2, 3, 128).float()), dict(v=half(2, 2, 2, 128)),
    dict(k_out=half(2, 2, 3, 128)), dict(q_out=half(2, 8, 3, 128), dtype=torch.float32), dict(q_out=half(2, 3, 8, 128).transpose(1, 2)), dict(q_out=half(2, 8, 4, 128)),
    dict(dtype=torch.float64), dict(n_new=ints(3)), dict(n_new=torch.zeros(2)), dict(first=ints(2, 3)), dict(depth=ints(2)), dict(depth=ints(2, 3).long()),
    dict(plan=None), dict(plan=[1.0])])
def test_rotary_checks_its_tensors(cache, plan, over):
    with pytest.raises(kv.KVLincError):
        cache.rotary(**{"plan": plan, "q": half(2, 8, 3, 128), **over})


MASS_TENSORS = [dict(mass=torch.zeros(2, 2, 2)), dict(mass=torch.zeros(2, 8, 3)), dict(mass=half(2, 2, 3)), dict(mass_out=torch.zeros(2, 2, 4)), dict(decay=-0.5),
                dict(decay=2.0), dict(decay=math.nan), dict(max_context=1 << 31), dict(mass=torch.zeros(2, 3, 2).transpose(1, 2))]


@pytest.mark.parametrize("over", MASS_TENSORS + [dict(q=half(2, 8, 1, 128)), dict(q=half(2, 2, 128)), dict(q=half(2, 8, 128).float()), dict(out=half(2, 2, 128)), dict(mass=None)])
def test_decode_mass_checks_its_tensors(cache, over):
    with pytest.raises(kv.KVLincError):
        cache.decode_mass(**{"q": half(2, 8, 128), "mass": torch.zeros(2, 2, 3), **over})


@pytest.mark.parametrize("over", MASS_TENSORS + [dict(q=half(2, 8, 128)), dict(q=half(2, 2, 4, 128)), dict(q=half(2, 8, 0, 128)), dict(n_rows=ints(3)), dict(n_rows=torch.zeros(2)),
                                                 dict(q=half(2, 4, 8, 128).transpose(1, 2))])
def test_attention_mass_checks_its_tensors(cache, over):
    with pytest.raises(kv.KVLincError):
        cache.attention_mass(**{"q": half(2, 8, 4, 128), "mass": torch.zeros(2, 2, 3), **over})


@pytest.mark.parametrize("over", [dict(mass=torch.zeros(2, 2, 2)), dict(mass=half(2, 2, 3)), dict(keep=-1), dict(keep=1 << 31), dict(limit=-1), dict(first=-1), dict(last=1 << 32),
                                  dict(mass_out=torch.zeros(2, 2, 4)), dict(offset=ints(3)), dict(offset=torch.zeros(2)), dict(offset_out=ints(1)), dict(kept=ints(2, 2, 3)),
                                  dict(to=3), dict(to="small"), dict(to="small", mass_out=torch.zeros(2, 2, 3)), dict(to="small", mass_out=torch.zeros(2, 2, 2), kept=ints(2, 2, 2))])
def test_evict_checks_its_tensors(cache, over):
    over = dict(over)
    if over.get("to") == "small":
        over["to"] = kv.KVLincCache(2, 8, 2, 128, device="cpu")
    with pytest.raises(kv.KVLincError):
        cache.evict(**{"mass": torch.zeros(2, 2, 3), "keep": 1, "first": 0, **over})


def test_a_cache_on_the_host_is_refused_last(cache, plan):
    for call in (lambda: cache.rotary(plan, half(2, 8, 3, 128)), lambda: cache.decode_mass(half(2, 8, 128), cache.new_mass()),
                 lambda: cache.attention_mass(half(2, 8, 3, 128)), lambda: cache.evict(cache.new_mass(), 2)):
        with pytest.raises(kv.KVLincError, match="GPU"):
            call()
