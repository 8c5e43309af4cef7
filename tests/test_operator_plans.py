"""CPU checks of the host code of the operators around a quantised layer (no GPU needed):
operator_check.cpp is compiled with hipcc against the library's sources."""
import os
import shutil
import subprocess

import pytest

from operator_sizes import BACKWARD, GATED, LINEAR_BIG

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    path = str(tmp_path_factory.mktemp("operators") / "operator_check")
    cmd = [hipcc, "-O1", "-std=c++17", "-w", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(ROOT, "paper_2608_06291_amd", "csrc"), "-o", path, os.path.join(HERE, "operator_check.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return path


@pytest.mark.timeout(300)
def test_launches_and_limits(exe):
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "fails 0" in r.stdout, r.stdout[-4000:]


def _plan(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0
    return tuple(int(v) for v in r.stdout.split())


def test_sizes_of_the_tile_tests_take_their_tiles(exe):
    """test_gpu_operators_tiles.py tests the 256 x 256 tiles only while its sizes take them."""
    for T, n, m in LINEAR_BIG:
        assert _plan(exe, "tile", m, T) == (256,), (T, n, m)
    for T, d, f in GATED:
        assert _plan(exe, "tile", 2 * f, T) == (256,), (T, d, f)
    # several chunks, odd numbers of them among these, the last not whole
    assert {3, 5, 7} <= {-(-n // 128) for _, n, _ in LINEAR_BIG} and {5, 7} <= {-(-d // 64) for _, d, _ in GATED}
    assert any(n % 128 for _, n, _ in LINEAR_BIG) and any(d % 64 for _, d, _ in GATED)
    seen = set()
    for T, d, f, _, _, dx, dw in BACKWARD:
        p = _plan(exe, "backward", T, d, f)
        assert (dx is None or p[:2] == dx) and (dw is None or p[2:] == dw), (T, d, f, p)
        seen |= {("dx", *(dx or ())), ("dw", *(dw or ()))}
    assert {("dx", 256, 1), ("dx", 256, 3), ("dw", 256, 1), ("dw", 256, 4)} <= seen
    # the gated product of the first of them, too (its rows are padded to whole chunks)
    T, _, f = BACKWARD[0][:3]
    assert _plan(exe, "tile", 2 * (-(-f // 64) * 64), T) == (256,)
