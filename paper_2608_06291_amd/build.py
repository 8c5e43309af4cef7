"""Build libbakron.so (hand-written HIP for gfx950) in-tree with hipcc."""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SOURCES = ["csrc/api.hip", "csrc/factor.hip", "csrc/solve.hip", "csrc/antidiag.hip",
           "csrc/hessian.hip", "csrc/quant.hip", "csrc/gptq.hip", "csrc/norm.hip", "csrc/linear.hip",
           "csrc/mlp.hip", "csrc/logprob.hip", "csrc/head.hip", "csrc/layernorm.hip", "csrc/embedding.hip"]
LIB = os.path.join(HERE, "libbakron.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # packed fp32 instructions are kept out of all device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result", "-Wno-unused-value",
]


def build(verbose: bool = False) -> str:
    """Compile every HIP source into paper_2608_06291_amd/libbakron.so."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB + ".tmp"
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    inc = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
        # (the host pass does not know the target feature: harmless)
        warnings = [w for w in res.stderr.splitlines(True) if "packed-fp32-ops" not in w]
        if warnings:
            sys.stderr.write("".join(warnings))

    # one object per source, side by side, then one link
    with tempfile.TemporaryDirectory() as obj, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(obj, os.path.basename(s) + ".o") for s in SOURCES]
        list(pool.map(run, [[hipcc, *flags, *inc, "-c", os.path.join(HERE, s), "-o", o]
                            for s, o in zip(SOURCES, objects)]))
        run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp, *objects])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
