"""The host side of kvlinc_bounded.h at the ends of its arguments' ranges, built so that a signed overflow ends the process."""
import os
import subprocess
import sys

import pytest

from tests.test_context_build import ROOT, build_module


@pytest.fixture(scope="module")
def checked_library(tmp_path_factory):
    build = build_module()
    if not all(os.path.exists(os.path.join(build.CSRC, n + ".o")) for n in build.LIBRARIES[build.LIB_PATH]):
        build.build()
    at = tmp_path_factory.mktemp("checked")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    obj, lib = str(at / "api.o"), str(at / "libchecked.so")
    check = ["-Xarch_host", "-fsanitize=signed-integer-overflow,shift", "-Xarch_host", "-fsanitize-trap=all"]  # (host code only)
    run = lambda *a: subprocess.run([hipcc, *a], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    run(*build.COMMON, *check, "-c", os.path.join(build.CSRC, "kvlinc_bounded_api.hip"), "-o", obj)
    others = [os.path.join(build.CSRC, n + ".o") for n in build.LIBRARIES[build.LIB_PATH] if n != "kvlinc_bounded_api"]
    run("--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib, obj, *others)
    return lib


CODE = """
import ctypes, itertools, sys
import torch  # (its copy of the HIP runtime serves the library)
import paper_2510_05373_amd.binding as kb
from tests.test_library_abi import fake_struct
L = ctypes.CDLL(sys.argv[1])
P, i32, size, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
for f in (L.kvlinc_decode_mass_workspace_bytes, L.kvlinc_attention_mass_workspace_bytes, L.kvlinc_cache_evict_workspace_bytes):
    f.restype = size
none = dict(S=0, S16=0, P=0, Wq=0, Wk=0)
top = 2 ** 31 - 1
shapes = [dict(B=b, H_q=h * g, H_kv=h, max_groups=m, bits=bits, **c) for b, h in ((1, 1), (1 << 12, 1 << 12), (1 << 24, 1), (1, (1 << 24) - 1), (1 << 20, 8))
          for g in (1, 8) for m in (1, 1024, 1025, 1 << 24, (1 << 24) - 4) for bits in (2, 4) for c in (none, {})]
plan = kb.RotationStruct(channels=128, interleaved=0, magnitude=1.0, freq=0x20000)
for s in shapes:
    c = fake_struct(**s)
    r = ctypes.byref(c)
    for bound in (0, 1, top, -top - 1):
        print(s, bound, file=sys.stderr)
        L.kvlinc_decode_mass_workspace_bytes(r, bound)
        # (no scratch, or an output that is an input: refused before a launch)
        assert L.kvlinc_decode_attention_mass(r, P(0x20000), P(0x20000), None, f32(1.0), P(0x20000), P(16), size(0), bound, None) == -1
        for T in (1, 1 << 20, (1 << 20) + 1, top, -1):
            L.kvlinc_attention_mass_workspace_bytes(r, T, bound)
            assert L.kvlinc_attention_mass(r, P(0x20000), None, T, None, f32(1.0), P(0x20000), P(16), size(0), bound, None) == -1
    L.kvlinc_cache_evict_workspace_bytes(r)
    for keep, limit, first, last in itertools.product((0, 1, top), (1, top), (0, 1, top), (0, 1, top)):
        assert L.kvlinc_cache_evict(r, r, P(0x20000), P(0x20004), keep, limit, first, last, None, None, None, P(16), size(0), None) < 0
    for T, stride, kind in itertools.product((1, 1 << 24, top), (0, 128, 1 << 48), (0, 1, 2)):
        rows = kb.RowsStruct(0x20000, 0x20010, stride, stride, stride)
        print(s, T, stride, kind, file=sys.stderr)
        # (rows moved by 16 bytes on themselves)
        assert L.kvlinc_rotary(r, ctypes.byref(plan), ctypes.byref(rows), None, None, T, None, None, None, 1, kind, kind, None) == -1
print("done")
"""


def test_no_signed_overflow(checked_library):
    r = subprocess.run([sys.executable, "-c", CODE, checked_library], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), (r.returncode, r.stderr[-800:])
