"""The host side of kvlinc_context.h at the ends of its arguments' ranges, built so that a signed overflow ends the process."""
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
    run(*build.COMMON, *check, "-c", os.path.join(build.CSRC, "kvlinc_context_api.hip"), "-o", obj)
    others = [os.path.join(build.CSRC, n + ".o") for n in build.LIBRARIES[build.LIB_PATH] if n != "kvlinc_context_api"]
    run("--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib, obj, *others)
    return lib


CODE = """
import ctypes, itertools, sys
import torch  # (its copy of the HIP runtime serves the library)
import paper_2510_05373_amd.binding as kb
from tests.test_library_abi import fake_struct
L = ctypes.CDLL(sys.argv[1])
P, i32, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
L.kvlinc_prompt_workspace_bytes.restype = L.kvlinc_decode_windowed_workspace_bytes.restype = size
none = dict(S=0, S16=0, P=0, Wq=0, Wk=0)
top = 2 ** 31 - 1
shapes = [dict(B=b, H_q=h * g, H_kv=h, max_groups=m, bits=bits, **c) for b, h in ((1, 1), (1 << 12, 1 << 12), (1 << 24, 1), (1, (1 << 24) - 1), (1 << 20, 8))
          for g in (1, 8) for m in (1, 1 << 24, (1 << 24) - 4) for bits in (2, 4) for c in (none, {})]
cells = ctypes.create_string_buffer(64)
for s in shapes:
    c = fake_struct(**s)
    r = ctypes.byref(c)
    for T, window, sinks, bound in itertools.product((1, 1 << 24, top), (0, 1, top), (0, top), (0, 1, top, -top - 1)):
        print(s, T, window, sinks, bound, file=sys.stderr)
        L.kvlinc_prompt_workspace_bytes(r, T, window, sinks, bound)
        L.kvlinc_decode_windowed_workspace_bytes(r, window, sinks, bound)
        # (an output that is its input, or no scratch: refused before a launch)
        assert L.kvlinc_prompt_attention(r, P(0x20000), P(0x20000), P(0x20000), None, T, window, sinks, P(0x20000), P(16), size(0), bound, None) == -1
    for T, dtype in itertools.product((1, 1 << 24, 1 << 30, top), (0, 1, 2)):
        print(s, T, dtype, file=sys.stderr)
        # (both outputs at one place)
        assert L.kvlinc_cache_read(r, None, T, P(0x20000), P(0x20000), dtype, 0, None) == -1
# more rows than a grid holds, whatever the outputs' places
c = fake_struct(B=1 << 24, H_q=1, H_kv=1, max_groups=1 << 24, **none)
for k, v in ((0x20000, 0x40000), (0x20000, None), (None, 0x20000), (0x20000, 1 << 62)):
    assert L.kvlinc_cache_read(ctypes.byref(c), None, 1 << 30, P(k), P(v), 2, 0, None) == -1
print("done")
"""


def test_no_signed_overflow(checked_library):
    r = subprocess.run([sys.executable, "-c", CODE, checked_library], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), (r.returncode, r.stderr[-800:])
