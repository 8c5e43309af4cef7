"""CPU checks of the built library: what build() shows, and that m0, which the assembly loads to LDS
write without being able to say so, is used for nothing else in their kernels."""
import glob
import os
import re
import struct
import subprocess
import types

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def _code_objects(path, tmp):
    """The gfx950 code objects that the library holds (offload bundles: a magic, a count, then offset,
    size and name of each entry)."""
    data, magic, at, out = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", 0, []
    while (at := data.find(magic, at)) >= 0:
        p = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + length] and size:
                f = str(tmp / f"{len(out)}.co")
                open(f, "wb").write(data[at + offset:at + offset + size])
                out.append(f)
            p += 24 + length
        at += 24
    return out


def test_m0_belongs_to_the_loads(tmp_path):
    import paper_2608_06291_amd as pk
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump not available")
    loads = 0
    for f in _code_objects(pk.LIB_PATH, tmp_path):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], capture_output=True, text=True).stdout
        for kernel in re.split(r"^[0-9a-f]+ <", text, flags=re.M)[1:]:
            if not re.match(r"_ZN2bk\d+(k_linear|k_gated|k_prod)", kernel):
                continue
            ins = [line.split("//")[0].strip() for line in kernel.splitlines()[1:] if line.strip()]
            for i, line in enumerate(ins):
                if re.search(r"\bm0\b", line):
                    assert line.startswith("s_mov_b32 m0, s") and ins[i + 1] == "s_nop 0", (kernel[:60], line)
                    assert ins[i + 2].startswith("global_load_lds_dword"), (kernel[:60], ins[i + 2])
                if "load_lds" in line:
                    assert ins[i - 2].startswith("s_mov_b32 m0, s"), (kernel[:60], line)
                    loads += 1
    assert loads > 500   # (the kernels were found)


def test_no_assembly_claims_a_reserved_register():
    for f in glob.glob(os.path.join(ROOT, "paper_2608_06291_amd", "csrc", "*")):
        for asm in re.findall(r"asm volatile\((.*?)\);", open(f).read(), flags=re.S):
            clobbers = asm.rsplit(":", 1)[-1]
            assert not re.search(r"\"(m0|exec|vcc|scc)\"", clobbers), (f, asm)


def test_build_shows_warnings(monkeypatch, capsys, tmp_path):
    from paper_2608_06291_amd import build
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build.os, "replace", lambda a, b: None)
    err = "a.hip:3: warning: something\nwarning: '-packed-fp32-ops' is not a recognized feature\n"
    monkeypatch.setattr(build.subprocess, "run", lambda *a, **k: types.SimpleNamespace(returncode=0, stdout="", stderr=err))
    build.build()
    shown = capsys.readouterr().err
    assert "warning: something" in shown and "packed" not in shown
