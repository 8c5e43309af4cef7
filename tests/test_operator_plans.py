"""CPU checks of the host code of the operators around a quantised layer (no GPU needed):
operator_check.cpp is compiled with hipcc against the library's sources."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("operators") / "operator_check")
    cmd = [hipcc, "-O1", "-std=c++17", "-w", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2608_06291_amd", "csrc"), "-o", exe, os.path.join(HERE, "operator_check.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return exe


@pytest.mark.timeout(300)
def test_launches_and_limits(checker):
    r = subprocess.run([checker], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "fails 0" in r.stdout, r.stdout[-4000:]
