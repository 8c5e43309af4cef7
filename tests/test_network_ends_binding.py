"""What the binding of the operators at the ends of a network keeps, and what it refuses before it looks at devices:
needs no GPU."""
import ctypes

import pytest

from test_network_ends_refusals import HEAD, HEAD_OK, HEADB, HEADB_OK, LNB, LNB_OK
from test_operators_refusals import P, _call, _size, lib  # noqa: F401


@pytest.mark.parametrize("name", ["bakron_head_logprobs", "bakron_head_logprobs_backward"])
def test_kept_sizes_of_head_calls(lib, name):  # noqa: F811
    """Calls that need workspaces of different sizes have different keys: each matrix alone and both with rows far apart, off
    an aligned start, at distances that are no multiples of 16 bytes."""
    import torch
    import paper_2608_06291_amd as pk
    names, base = (HEAD, HEAD_OK) if name == "bakron_head_logprobs" else (HEADB, dict(HEADB_OK, dw=P))
    dev, T, d, V = torch.device("cuda", 0), 40, 64, 5000
    sizes = {}
    far = ((4096, 64), (4096, 1 << 22), (4096, (1 << 22) + 8), (4098, 64), (4096, 65), (4096, 1 << 30))
    for xp, ldx in far:
        for wp, ldw in far:
            need = ctypes.c_size_t(0)
            assert _call(getattr(lib, name), names, dict(base, T=T, d=d, V=V, x=ctypes.c_void_p(xp), ldx=ldx, w=ctypes.c_void_p(wp), ldw=ldw, work=None,
                                                         size=ctypes.byref(need))) == 0
            key = pk._lib._head_key(name, dev, xp, ldx, T, d, wp, ldw, V)
            assert sizes.setdefault(key, need.value) == need.value, (xp, ldx, wp, ldw)
    assert len(set(sizes.values())) == 4   # (none copied, x, w, both)


class _Rows:
    """As much of a tensor as the binding looks at."""

    def __init__(self, device, *shape):
        import torch
        self.shape, self.dtype, self.device, self.requires_grad = shape, torch.bfloat16, device, False


def test_kept_sizes_of_norm_gradients(monkeypatch):
    """The size depends on the CUs of the device: each device has its own."""
    import torch
    import paper_2608_06291_amd as pk
    keys = []
    monkeypatch.setattr(pk._lib, "_rows_of", lambda t, *more: (4096, t.shape[1]))
    monkeypatch.setattr(pk._lib, "_vector", lambda *more: 4096)
    monkeypatch.setattr(pk._lib, "_run_op", lambda fn, args, device, work=None, key=None: keys.append(key))

    class Torch:
        def __getattr__(self, name):
            return (lambda *shape, **more: _Rows(more["device"], *shape)) if name == "empty" else getattr(torch, name)
    monkeypatch.setattr(_Rows, "data_ptr", lambda self: 4096, raising=False)
    pk._lib._import_torch()
    monkeypatch.setattr(pk._lib, "_torch", Torch())
    for index in (0, 1):
        x = _Rows(torch.device("cuda", index), 50, 8)
        pk.layernorm_backward(x, x, None, None, None)
    assert len(keys) == 2 and keys[0] != keys[1]


def test_outputs_that_require_gradients():
    """An output that autograd follows is not overwritten silently."""
    import torch
    import paper_2608_06291_amd as pk
    x, tok = torch.zeros((2, 4)), torch.zeros(2, dtype=torch.int64)
    out, table = torch.zeros((2, 4), requires_grad=True), torch.zeros((3, 4), requires_grad=True)
    for call in (lambda: pk.layernorm(x, sum_out=out), lambda: pk.layernorm(x, residual=x, sum_out=out), lambda: pk.embedding(tok, x, out=out),
                 lambda: pk.embedding_backward(x, tok, 3, out=table), lambda: pk.embedding_backward(x, tok, 3, base=table, out=table)):
        with pytest.raises(RuntimeError, match="no_grad"):
            call()
        with torch.no_grad(), pytest.raises(TypeError, match="CUDA"):   # (taken, but for the device)
            call()


@pytest.mark.parametrize("name,ld", [("dy", "lddy"), ("x", "ldx"), ("ds", "ldds")])
def test_norm_gradients_in_place_need_the_same_rows(lib, name, ld):  # noqa: F811
    base = dict(LNB_OK, size=_size(1 << 50), dy=ctypes.c_void_p(16384), x=ctypes.c_void_p(32768), ds=ctypes.c_void_p(65536), dw=P)
    base["dx"] = base[name]
    assert _call(lib.bakron_layernorm_backward, LNB, dict(base, T=0, dw=None)) == 0
    assert _call(lib.bakron_layernorm_backward, LNB, base, **{ld: 72}) == 1
    assert b"in place" in lib.bakron_last_error()
