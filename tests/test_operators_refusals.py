"""What the operators around a quantised layer refuse, on the host and before any work:
needs no GPU (the pointers are never followed)."""
import ctypes
import math

import pytest

P = ctypes.c_void_p(4096)
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    import paper_2608_06291_amd as pk
    return pk.load()


def _size(n=0):
    return ctypes.byref(ctypes.c_size_t(n))


def _call(fn, names, base, **change):
    args = dict(base, **change)
    assert set(change) <= set(names), change
    return fn(*[args[n] for n in names])


NORM = "x ldx residual ldr dtype T d weight eps normalise sum lds y ldy q ldq scale stream".split()
NORM_OK = dict(x=P, ldx=64, residual=P, ldr=64, dtype=BF16, T=0, d=64, weight=None, eps=1e-5, normalise=1,
               sum=None, lds=64, y=None, ldy=64, q=P, ldq=128, scale=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(T=1 << 31), dict(d=0), dict(d=65537, ldx=1 << 17), dict(dtype=3), dict(dtype=-1),
    dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(scale=None), dict(q=None), dict(ldx=63),
    dict(ldr=63), dict(ldq=63), dict(sum=P, lds=63), dict(y=P, ldy=1), dict(sum=P, lds=65), dict(T=1, x=None)])
def test_norm_refuses(lib, change):
    assert _call(lib.bakron_rmsnorm_quant, NORM, NORM_OK) == 0
    assert _call(lib.bakron_rmsnorm_quant, NORM, NORM_OK, **change) == 1
    assert b"bakron_rmsnorm_quant" in lib.bakron_last_error()


@pytest.mark.parametrize("args", [(P, 0, 5, 4, P), (P, 5, 0, 4, P), (P, 5, (1 << 17) + 1, 4, P), (P, (1 << 20) + 1, 5, 4, P),
                                  (P, 5, 5, 3, P), (None, 5, 5, 4, P), (P, 5, 5, 8, None), (P, 5, 5, 8, ctypes.c_void_p(4104))])
def test_pack_refuses(lib, args):
    assert lib.bakron_pack_codes(*args, None) == 1
    assert b"bakron_pack_codes" in lib.bakron_last_error()


LINEAR = ("q ldq q_scale T n packed width m scale group bias act other ldo combine y ldy dtype work size "
          "stream").split()
LINEAR_OK = dict(q=P, ldq=128, q_scale=None, T=0, n=100, packed=P, width=4, m=10, scale=P, group=64, bias=None,
                 act=0, other=None, ldo=10, combine=0, y=P, ldy=10, dtype=BF16, work=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(n=0), dict(n=(1 << 17) + 1), dict(m=0), dict(m=(1 << 20) + 1), dict(width=5), dict(group=-64),
    dict(group=32), dict(group=100), dict(act=3), dict(act=-1), dict(combine=3), dict(combine=1), dict(other=P),
    dict(ldq=127), dict(ldq=136), dict(ldq=100), dict(ldy=9), dict(other=P, combine=1, ldo=9), dict(dtype=7),
    dict(other=P, combine=1, ldo=11), dict(T=1, q=None), dict(T=1, scale=None), dict(T=1, y=None),
    dict(T=1, q=ctypes.c_void_p(4104)), dict(T=1, packed=ctypes.c_void_p(4104)), dict(T=(1 << 31) - 1, m=1 << 20, ldy=1 << 20)])
def test_linear_refuses(lib, change):
    base = dict(LINEAR_OK, size=_size())
    assert _call(lib.bakron_linear, LINEAR, base) == 0
    assert _call(lib.bakron_linear, LINEAR, base, **change) == 1
    assert b"bakron_linear" in lib.bakron_last_error()
    assert _call(lib.bakron_linear, LINEAR, dict(base, size=None)) == 1


MLP = "x ldx T d wg wu ldw f dtype act h ldh fu fg work size stream".split()
MLP_OK = dict(x=P, ldx=64, T=0, d=64, wg=P, wu=P, ldw=64, f=32, dtype=BF16, act=1, h=P, ldh=32, fu=None, fg=None,
              work=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(d=0), dict(f=0), dict(d=(1 << 17) + 1, ldx=1 << 18, ldw=1 << 18), dict(f=(1 << 17) + 1, ldh=1 << 18),
    dict(ldx=63), dict(ldw=63), dict(ldh=31), dict(dtype=F32), dict(dtype=5), dict(act=0), dict(act=3), dict(T=1, x=None),
    dict(T=1, wg=None), dict(T=1, wu=None), dict(T=1, h=None), dict(T=1 << 40)])
def test_mlp_refuses(lib, change):
    base = dict(MLP_OK, size=_size())
    assert _call(lib.bakron_gated_mlp, MLP, base) == 0
    assert _call(lib.bakron_gated_mlp, MLP, base, **change) == 1
    assert b"bakron_gated_mlp" in lib.bakron_last_error()


BWD = "dh lddh x ldx T d wg wu ldw f dtype act dx lddx dwg dwu lddw work size stream".split()
BWD_OK = dict(dh=P, lddh=32, x=P, ldx=64, T=0, d=64, wg=P, wu=P, ldw=64, f=32, dtype=F16, act=2, dx=P, lddx=64,
              dwg=None, dwu=None, lddw=64, work=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(lddh=31), dict(lddx=63), dict(dwg=P, dwu=P, lddw=63), dict(dwg=P), dict(dwu=P), dict(dx=None), dict(act=0),
    dict(dtype=F32), dict(T=1, dh=None), dict(T=1, x=None), dict(T=-1)])
def test_mlp_backward_refuses(lib, change):
    base = dict(BWD_OK, size=_size(1 << 40))
    assert _call(lib.bakron_gated_mlp_backward, BWD, base) == 0
    assert _call(lib.bakron_gated_mlp_backward, BWD, base, **change) == 1
    assert b"bakron_gated_mlp_backward" in lib.bakron_last_error()


def test_mlp_backward_workspace(lib):
    base = dict(BWD_OK, T=100)
    need = ctypes.c_size_t(0)
    assert _call(lib.bakron_gated_mlp_backward, BWD, dict(base, work=None, size=ctypes.byref(need))) == 0
    assert need.value > 0
    assert _call(lib.bakron_gated_mlp_backward, BWD, dict(base, size=_size(need.value - 1))) == 1
    assert b"too small" in lib.bakron_last_error()
    assert _call(lib.bakron_gated_mlp_backward, BWD, dict(base, work=ctypes.c_void_p(4104), size=_size(need.value))) == 1
    assert b"aligned" in lib.bakron_last_error()


LP = "z ld dtype T V target top logprob entropy lse tl ti work size stream".split()
LP_OK = dict(z=P, ld=100, dtype=F32, T=0, V=100, target=P, top=0, logprob=P, entropy=P, lse=P, tl=None, ti=None,
             work=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(V=0), dict(V=(1 << 20) + 1, ld=1 << 21), dict(ld=99), dict(dtype=3), dict(top=-1), dict(top=33),
    dict(top=5), dict(top=5, tl=P), dict(top=5, ti=P), dict(tl=P, ti=P), dict(target=None), dict(V=4, top=5, tl=P, ti=P),
    dict(T=1, z=None), dict(T=1 << 30)])
def test_logprobs_refuse(lib, change):
    base = dict(LP_OK, size=_size(1 << 50))
    assert _call(lib.bakron_token_logprobs, LP, base) == 0
    assert _call(lib.bakron_token_logprobs, LP, base, **change) == 1
    assert b"bakron_token_logprobs" in lib.bakron_last_error()


LPB = "z ld dtype T V target lse entropy gl gh d ldd stream".split()
LPB_OK = dict(z=P, ld=100, dtype=F16, T=0, V=100, target=P, lse=P, entropy=P, gl=P, gh=P, d=P, ldd=100, stream=None)


@pytest.mark.parametrize("change", [
    dict(T=-1), dict(V=0), dict(ld=99), dict(ldd=99), dict(ldd=101), dict(dtype=9), dict(target=None), dict(entropy=None),
    dict(T=1, z=None), dict(T=1, lse=None), dict(T=1, d=None), dict(T=1 << 30)])
def test_logprobs_backward_refuse(lib, change):
    assert _call(lib.bakron_token_logprobs_backward, LPB, LPB_OK) == 0
    assert _call(lib.bakron_token_logprobs_backward, LPB, LPB_OK, **change) == 1
    assert b"bakron_token_logprobs_backward" in lib.bakron_last_error()


def test_binding_refuses():
    import torch
    import paper_2608_06291_amd as pk
    with pytest.raises(TypeError):
        pk.rmsnorm_quant(torch.zeros((2, 4)))
    with pytest.raises(TypeError):
        pk.gated_mlp(torch.zeros((2, 4)), torch.zeros((3, 4)), torch.zeros((3, 4)))
    with pytest.raises(TypeError):
        pk.token_logprobs(torch.zeros((2, 4)))
    with pytest.raises(TypeError):
        pk.pack_codes(torch.zeros((2, 4), dtype=torch.int8))
