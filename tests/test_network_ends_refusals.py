"""What the operators at the ends of a network refuse, on the host and before any work: needs no
GPU (the pointers are never followed)."""
import ctypes
import math

import pytest

from test_operators_refusals import BF16, F16, F32, P, _call, _size, lib  # noqa: F401

BIG = 1 << 50
HEAD = "x ldx T d w ldw V dtype target logprob entropy lse work size stream".split()
HEAD_OK = dict(x=P, ldx=64, T=0, d=64, w=P, ldw=64, V=100, dtype=BF16, target=P, logprob=P, entropy=P, lse=P, work=P, stream=None)
HEADB = "x ldx T d w ldw V dtype target lse entropy gl gh dx lddx dw lddw work size stream".split()
HEADB_OK = dict(x=P, ldx=64, T=0, d=64, w=P, ldw=64, V=100, dtype=F16, target=P, lse=P, entropy=P, gl=P, gh=P, dx=P, lddx=64,
                dw=None, lddw=64, work=P, stream=None)
LN = "x ldx residual ldr dtype T d weight bias eps centre sum lds y ldy mean rstd stream".split()
LN_OK = dict(x=P, ldx=64, residual=P, ldr=64, dtype=BF16, T=0, d=64, weight=P, bias=P, eps=1e-5, centre=1,
             sum=ctypes.c_void_p(8192), lds=64, y=P, ldy=64, mean=P, rstd=P, stream=None)
LNB = "dy lddy x ldx dtype T d weight mean rstd ds ldds dx lddx dw db work size stream".split()
LNB_OK = dict(dy=P, lddy=64, x=P, ldx=64, dtype=F32, T=0, d=64, weight=P, mean=P, rstd=P, ds=ctypes.c_void_p(8192), ldds=64, dx=P, lddx=64,
              dw=None, db=None, work=P, stream=None)
EMB = "tokens T table ldt dtype V d scale y ldy stream".split()
EMB_OK = dict(tokens=P, T=0, table=P, ldt=64, dtype=F16, V=10, d=64, scale=1.0, y=P, ldy=64, stream=None)
EMBB = "dy lddy tokens T dtype V d scale onto ldb out ldo work size stream".split()
EMBB_OK = dict(dy=P, lddy=64, tokens=P, T=1, dtype=F16, V=10, d=64, scale=1.0, onto=P, ldb=64, out=ctypes.c_void_p(8192), ldo=64,
               work=P, stream=None)

SIZES = [dict(T=-1), dict(T=1 << 31), dict(T=(1 << 63) - 1), dict(d=0), dict(dtype=3), dict(dtype=-1), dict(size=None)]


@pytest.mark.parametrize("change", SIZES + [
    dict(d=65), dict(ldw=63), dict(ldx=63), dict(V=0), dict(V=(1 << 20) + 1), dict(d=(1 << 17) + 1, ldx=1 << 18, ldw=1 << 18), dict(dtype=F32),
    dict(target=None), dict(T=1, x=None), dict(T=1, w=None), dict(T=1, logprob=None, entropy=None, lse=None), dict(T=(1 << 27) + 1, V=1),
    dict(T=1 << 26, V=1 << 12), dict(T=100, size=_size(100)), dict(T=100, work=ctypes.c_void_p(4104))])
def test_head_refuses(lib, change):  # noqa: F811
    base = dict(HEAD_OK, size=_size(BIG))
    assert _call(lib.bakron_head_logprobs, HEAD, base) == 0
    assert _call(lib.bakron_head_logprobs, HEAD, base, **change) == 1
    assert b"bakron_head_logprobs" in lib.bakron_last_error()


@pytest.mark.parametrize("change", SIZES + [
    dict(d=65), dict(ldw=63), dict(ldx=63), dict(lddx=63), dict(dw=P, lddw=63), dict(V=0), dict(V=(1 << 20) + 1), dict(dtype=F32),
    dict(target=None), dict(entropy=None), dict(dx=None), dict(T=1, x=None), dict(T=1, w=None), dict(T=1, lse=None), dict(T=1 << 26, V=1 << 12),
    dict(T=100, size=_size(100))])
def test_head_backward_refuses(lib, change):  # noqa: F811
    base = dict(HEADB_OK, size=_size(BIG))
    assert _call(lib.bakron_head_logprobs_backward, HEADB, base) == 0
    assert _call(lib.bakron_head_logprobs_backward, HEADB, base, **change) == 1
    assert b"bakron_head_logprobs_backward" in lib.bakron_last_error()


@pytest.mark.parametrize("change", SIZES[:-1] + [
    dict(d=65537, ldx=1 << 17, ldr=1 << 17, lds=1 << 17, ldy=1 << 17), dict(eps=0.0), dict(eps=-1.0), dict(eps=9e-31), dict(eps=math.nan),
    dict(eps=math.inf), dict(ldx=63), dict(ldr=63), dict(lds=63), dict(ldy=63), dict(sum=P, lds=65), dict(centre=0), dict(T=1, x=None),
    dict(T=1, sum=None, y=None, mean=None, rstd=None), dict(T=1 << 26)])
def test_layernorm_refuses(lib, change):  # noqa: F811
    assert _call(lib.bakron_layernorm, LN, LN_OK) == 0
    assert _call(lib.bakron_layernorm, LN, LN_OK, **change) == 1
    assert b"bakron_layernorm" in lib.bakron_last_error()


@pytest.mark.parametrize("change", SIZES + [
    dict(d=65537, ldx=1 << 17, lddy=1 << 17, ldds=1 << 17, lddx=1 << 17), dict(lddy=63), dict(ldx=63), dict(ldds=63), dict(lddx=63),
    dict(ds=P, ldds=65), dict(dx=None), dict(T=1, dy=None), dict(T=1, x=None), dict(T=1, rstd=None), dict(T=1 << 26),
    dict(T=50, dw=P, size=_size(10)), dict(T=50, db=P, work=ctypes.c_void_p(4104))])
def test_layernorm_backward_refuses(lib, change):  # noqa: F811
    base = dict(LNB_OK, size=_size(BIG))
    assert _call(lib.bakron_layernorm_backward, LNB, base) == 0
    assert _call(lib.bakron_layernorm_backward, LNB, base, **change) == 1
    assert b"bakron_layernorm_backward" in lib.bakron_last_error()


@pytest.mark.parametrize("change", SIZES[:-1] + [
    dict(T=(1 << 20) + 1), dict(V=0), dict(V=(1 << 20) + 1), dict(d=65537, ldt=1 << 17, ldy=1 << 17), dict(ldt=63), dict(ldy=63),
    dict(T=1, tokens=None), dict(T=1, table=None), dict(T=1, y=None), dict(T=1 << 20, d=65536, ldt=65536, ldy=65536, dtype=F32)])
def test_embedding_refuses(lib, change):  # noqa: F811
    assert _call(lib.bakron_embedding, EMB, EMB_OK) == 0
    assert _call(lib.bakron_embedding, EMB, EMB_OK, **change) == 1
    assert b"bakron_embedding" in lib.bakron_last_error()


@pytest.mark.parametrize("change", SIZES + [
    dict(T=(1 << 20) + 1), dict(V=0), dict(V=(1 << 20) + 1), dict(d=65537, lddy=1 << 17, ldb=1 << 17, ldo=1 << 17), dict(lddy=63), dict(ldb=63),
    dict(ldo=63), dict(onto=ctypes.c_void_p(8192), ldb=65), dict(out=None), dict(dy=None), dict(tokens=None), dict(T=1000, size=_size(10)),
    dict(T=1000, work=ctypes.c_void_p(4104))])
def test_embedding_backward_refuses(lib, change):  # noqa: F811
    base = dict(EMBB_OK, size=_size(BIG))
    assert _call(lib.bakron_embedding_backward, EMBB, base, **change) == 1
    assert b"bakron_embedding_backward" in lib.bakron_last_error()


@pytest.mark.parametrize("name", ["bakron_head_logprobs", "bakron_head_logprobs_backward", "bakron_layernorm_backward",
                                  "bakron_embedding_backward"])
def test_workspace_sizes(lib, name):  # noqa: F811
    """What is asked for is enough, and one byte less is not."""
    names, base = {"bakron_head_logprobs": (HEAD, HEAD_OK), "bakron_head_logprobs_backward": (HEADB, dict(HEADB_OK, dw=P)),
                   "bakron_layernorm_backward": (LNB, dict(LNB_OK, dw=P)), "bakron_embedding_backward": (EMBB, EMBB_OK)}[name]
    fn = getattr(lib, name)
    for T in (1, 40, 700, 20000):
        need = ctypes.c_size_t(0)
        assert _call(fn, names, dict(base, T=T, work=None, size=ctypes.byref(need))) == 0
        if T <= {"bakron_embedding_backward": 256, "bakron_layernorm_backward": 32}.get(name, 0):
            assert need.value == 0
            continue
        assert need.value > 0
        assert _call(fn, names, dict(base, T=T, size=_size(need.value - 1))) == 1
        assert b"too small" in lib.bakron_last_error()


def test_binding_refuses():
    import torch
    import paper_2608_06291_amd as pk
    x, w, t = torch.zeros((2, 4), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: pk.head_logprobs(x, w, t), lambda: pk.head_logprobs_backward(x, w, t, torch.zeros(2)),
                 lambda: pk.layernorm(x), lambda: pk.layernorm_backward(x, x, None, None, torch.zeros(2)),
                 lambda: pk.embedding(t, w), lambda: pk.embedding_backward(x, t, 3)):
        with pytest.raises(TypeError):
            call()
