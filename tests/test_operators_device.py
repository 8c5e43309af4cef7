"""The library launches on the current device, so the binding makes that of the tensors current for
a call.  Needs no GPU: torch and the library are stood in for by objects that record."""
import contextlib
import ctypes
import types

import pytest


class _Machine:
    """Two devices, 0 being current; each with a stream of its own."""

    def __init__(self):
        self.current = 0
        self.calls = []
        self._C = types.SimpleNamespace(_cuda_getDevice=lambda: self.current, _cuda_getCurrentRawStream=lambda i: 1000 + i)
        self.cuda = types.SimpleNamespace(device=self._device, current_device=lambda: self.current)
        self.uint8 = None

    @contextlib.contextmanager
    def _device(self, device):
        before, self.current = self.current, device.index
        try:
            yield
        finally:
            self.current = before

    def empty(self, need, dtype, device):
        return types.SimpleNamespace(is_cuda=True, device=device, is_contiguous=lambda: True, data_ptr=lambda: 512,
                                     numel=lambda: need, element_size=lambda: 1)

    def operator(self, need):
        """A library function that needs so much workspace."""
        def fn(*args):
            self.calls.append((self.current, args))
            if len(args) > 2:
                work, size = args[-3], args[-2]
                if work is None:
                    size.value = need
                elif size.value < need:
                    return 1
            return 0
        return fn


@pytest.fixture
def machine(monkeypatch):
    from paper_2608_06291_amd import _lib
    m = _Machine()
    monkeypatch.setattr(_lib, "_torch", m)
    return m


def _device(index):
    return types.SimpleNamespace(type="cuda", index=index)


@pytest.mark.parametrize("index", [0, 1])
def test_calls_without_workspace(machine, index):
    from paper_2608_06291_amd import _lib
    _lib._run(machine.operator(0), (7,), _device(index))
    assert machine.calls == [(index, (7, 1000 + index))] and machine.current == 0


@pytest.mark.parametrize("index", [0, 1])
@pytest.mark.parametrize("need", [0, 4096])
@pytest.mark.parametrize("maybe_none", [True, False])
def test_calls_with_workspace(machine, index, need, maybe_none):
    from paper_2608_06291_amd import _lib
    _lib._run_op(machine.operator(need), (7,), _device(index), maybe_none=maybe_none)
    assert machine.current == 0
    assert all(c[0] == index and c[1][0] == 7 and c[1][-1] == 1000 + index for c in machine.calls)
    work, size = machine.calls[-1][1][1:3]
    assert work is not None and size.value >= need


def test_calls_of_the_solver(monkeypatch):
    """Every other call, and the methods of a factor that launch: the first tensor's device."""
    import torch
    import paper_2608_06291_amd as pk
    m = _Machine()
    monkeypatch.setattr(torch.cuda, "device", m._device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: m.current)
    seen = []

    class Stop(Exception):
        pass

    class Tensor:
        device = _device(1)

        def __getattr__(self, name):   # what a call asks of its tensor first
            seen.append(m.current)
            raise Stop

    def stop(*args):
        seen.append(m.current)
        raise Stop
    monkeypatch.setattr(pk._lib, "_check_dev", stop)
    monkeypatch.setattr(pk._lib, "_stream", stop)
    t = Tensor()
    calls = [lambda: pk.factor(t, None, 0.1), lambda: pk.solve(t, None, 4, None), lambda: pk.solve_noalloc(t, None, 4, None),
             lambda: pk.solve_antidiag(t, None, 4, None), lambda: pk.factor_blockdiag(t, None, 0.1),
             lambda: pk.mse_scales(t, 4), lambda: pk.gram(t), lambda: pk.gram(X=t), lambda: pk.sample_weights(t),
             lambda: pk.quadform_weights(t, None), lambda: pk.kron_factors(t, t), lambda: pk.mlp_local_factors(t, t, t)]
    f = pk.Factors.__new__(pk.Factors)
    f._h, f.n, f.m, f.device = ctypes.c_void_p(0), 0, 0, _device(1)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: stop())
    calls += [lambda: f.export("A"), f.check]
    for call in calls:
        before = len(seen)
        with pytest.raises(Stop):
            call()
        assert len(seen) > before and set(seen[before:]) == {1} and m.current == 0
