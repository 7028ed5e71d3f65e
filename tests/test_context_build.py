"""What the compiler makes of the kernels' inline assembly, looked at on the host: waits that the hardware leaves to the program."""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUILD = os.path.join(ROOT, "paper_2510_05373_amd", "build.py")


def build_module():
    spec = importlib.util.spec_from_file_location("kvlinc_build_by_path", BUILD)
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    return build


def assembly(source, tmp_path):
    build = build_module()
    out = tmp_path / (source + ".s")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    r = subprocess.run([hipcc, *build.COMMON, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    lines = (re.sub(r";.*", "", line).strip() for line in out.read_text().splitlines())
    return [line for line in lines if line and not line.startswith(".")]


def registers(text):
    """Scalar registers that a list of operands names."""
    found = set()
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        found.update(range(int(a), int(b) + 1))
    found.update(int(n) for n in re.findall(r"\bs(\d+)\b", text))
    return found


def states(line):
    """Wait states of an instruction."""
    op, _, rest = line.partition(" ")
    return int(rest, 0) + 1 if op == "s_nop" else 1


@pytest.mark.parametrize("source", ["kvlinc_dense.hip"])
def test_loads_into_lds_keep_their_distance(source, tmp_path):
    # A load that writes LDS takes its place there from m0: one wait state after a scalar write of m0.  Its base comes from scalar registers: five after
    # a vector instruction that writes one of them.
    code = assembly(source, tmp_path)
    loads = [i for i, line in enumerate(code) if re.match(r"(global|buffer|scratch)_load_(lds_\w+|.*\blds\b)", line)]
    assert loads
    for i in loads:
        base, gone = registers(code[i].partition(" ")[2]), 0
        for line in reversed(code[:i]):
            if line.endswith(":") or gone >= 5:
                break
            op, _, rest = line.partition(" ")
            target = rest.split(",")[0]
            if op.startswith("s_") and target.strip() == "m0":
                assert gone >= 1, (line, code[i])
            if op.startswith("v_") and not op.startswith("v_mfma"):
                assert not registers(target) & base, (line, code[i])
            gone += states(line)


def test_the_plan_and_the_joins_share_their_largest_number_of_splits():
    # (a row's join has room for 32 weights in LDS and reads two splits a lane)
    csrc = os.path.join(ROOT, "paper_2510_05373_amd", "csrc")
    text = "".join(open(os.path.join(csrc, f)).read() for f in sorted(os.listdir(csrc)) if f.endswith((".h", ".hip")))
    assert re.findall(r"constexpr int kMaxContextSplits = (\d+);", text) == ["32"]
    from paper_2510_05373_amd import binding as kb
    from tests.test_library_abi import fake_struct
    none = dict(S=0, S16=0, P=0, Wq=0, Wk=0)
    longest = fake_struct(B=1, H_q=1, H_kv=1, max_groups=1 << 20, **none)
    part = 132 * 4  # bytes of a split's partial result
    assert kb.kvlinc_prompt_workspace_bytes(longest, 1) == 32 * part
    assert kb.kvlinc_prompt_workspace_bytes(longest, 100) == 32 * part * 100
    assert kb.kvlinc_decode_windowed_workspace_bytes(longest, 0) == 32 * part
