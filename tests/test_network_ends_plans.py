"""CPU checks of the host code of the operators at the ends of a network (no GPU needed):
network_ends_check.cpp is compiled with hipcc against the library's sources; and m0 in the kernels that load
to LDS in assembly."""
import os
import re
import shutil
import subprocess

import pytest

from network_ends_sizes import HEAD, HEAD_LARGE
from test_build import OBJDUMP, _code_objects

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    path = str(tmp_path_factory.mktemp("ends") / "network_ends_check")
    cmd = [hipcc, "-O1", "-std=c++17", "-w", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2608_06291_amd", "csrc"), "-o", path, os.path.join(HERE, "network_ends_check.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return path


@pytest.mark.timeout(300)
def test_launches_and_limits(exe):
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    bad = [line for line in r.stdout.splitlines() if not line.startswith("ok")]
    assert r.returncode == 0 and "fails 0" in r.stdout, bad[:20]


def test_sizes_take_their_kernels(exe):
    """The sizes of test_gpu_network_ends.py take every kernel and tile of the vocabulary loss."""
    kinds, seen, pieces, columns = set(), set(), set(), set()
    for T, d, V, _, _ in HEAD + HEAD_LARGE:
        kind, n, dx, dx_parts, dw, dw_parts, tp = map(int, subprocess.run(
            [exe, "head", str(T), str(d), str(V)], capture_output=True, text=True, timeout=100).stdout.split())
        kinds.add(kind)
        pieces.add(min(n, 3))
        columns.add(tp > 0)
        if T > 32:
            seen |= {("dx", dx, dx_parts > 1), ("dw", dw, dw_parts > 1)}
    assert {-4, -2, -1, 64, 128, 256} <= kinds and {1, 2, 3} <= pieces and columns == {True, False}
    assert {("dx", 256, False), ("dx", 128, True), ("dx", 64, True), ("dx", 64, False), ("dw", 256, False), ("dw", 128, True),
            ("dw", 128, False), ("dw", 64, False)} <= seen, seen


def test_m0_belongs_to_the_loads(tmp_path):
    import paper_2608_06291_amd as pk
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump not available")
    loads = 0
    for f in _code_objects(pk.LIB_PATH, tmp_path):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], capture_output=True, text=True).stdout
        for kernel in re.split(r"^[0-9a-f]+ <", text, flags=re.M)[1:]:
            if not re.match(r"_ZN2bk\d+k_head", kernel):
                continue
            ins = [line.split("//")[0].strip() for line in kernel.splitlines()[1:] if line.strip()]
            for i, line in enumerate(ins):
                if re.search(r"\bm0\b", line):
                    assert line.startswith("s_mov_b32 m0, s") and ins[i + 1] == "s_nop 0", (kernel[:60], line)
                    assert ins[i + 2].startswith("global_load_lds_dword"), (kernel[:60], ins[i + 2])
                if "load_lds" in line:
                    assert ins[i - 2].startswith("s_mov_b32 m0, s"), (kernel[:60], line)
                    loads += 1
    assert loads > 100   # (the kernels were found)
