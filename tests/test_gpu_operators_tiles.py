"""GPU tests of the tiles that carry the large products, at sizes that reach them:
256 x 256 and 128 x 128 tiles over several chunks of the summed axis, an odd number of them and a last
one that is not whole, products cut into parts, operands in two pieces.

Which tile a size takes is asserted on the CPU (test_operator_plans.py, from the same lists).
References are 64-bit products, made on the GPU; tolerances as in test_gpu_operators.py.
"""
import pytest

from operator_sizes import BACKWARD, GATED, LINEAR_BIG
from test_gpu_operators import U32, _act64, _dtype, _gen, _say, _slope64, _t, _tiny, _u

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inside(got, want, tol, label):
    torch = _t()
    err = (got.double() - want).abs()
    bad = ~(err <= tol)   # (NaN is bad)
    assert not bool(bad.any()), (label, int(bad.sum()), float((err / tol).max()))


def _rand(shape, seed, scale=1.0):
    torch = _t()
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * scale


def _rows8(T, n):
    torch = _t()
    g = torch.Generator(device=DEV).manual_seed(T + n)
    q = torch.full((T, -(-n // 128) * 128), 99, dtype=torch.int8, device=DEV)   # (padding counts for nothing)
    q[:, :n] = torch.randint(-127, 128, (T, n), generator=g, device=DEV, dtype=torch.int8)
    return q[:, :n]


@pytest.mark.parametrize("T,n,m", LINEAR_BIG)
@pytest.mark.parametrize("width", [4, 8])
def test_linear_tiles_are_exact(T, n, m, width):
    """Sums below 2^24 and scales that are powers of two: every bit is determined."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear tiles", T, n, m, width)
    q = _rows8(T, n)
    c = torch.randint(-8 if width == 4 else -128, 8 if width == 4 else 128, (m, n), dtype=torch.int8, device=DEV,
                      generator=torch.Generator(device=DEV).manual_seed(3))
    y = pk.linear(q, torch.full((T,), 0.25, device=DEV), pk.pack_codes(c, width), torch.full((m,), 0.5, device=DEV),
                  dtype=torch.float32)
    want = q.double() @ c.double().t()
    assert float(want.abs().max()) < 2 ** 24
    assert torch.equal(y.double(), want * 0.125)


@pytest.mark.parametrize("T,n,m", LINEAR_BIG[:2])
@pytest.mark.parametrize("width,act,combine,dtype", [(4, "silu", "mul", "bf16"), (4, "gelu", "add", "f16"),
                                                     (8, "gelu", "mul", "bf16"), (8, "silu", "add", "f32")])
def test_linear_tiles_with_epilogue(T, n, m, width, act, combine, dtype):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear tiles, epilogue", T, n, m, width, act, combine, dtype)
    dt = _dtype(dtype)
    q = _rows8(T, n)
    top = 7 if width == 4 else 127
    c = torch.randint(-top, top + 1, (m, n), dtype=torch.int8, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4))
    scale = (1 + _rand((m,), 5).abs()) / (top * 64 * n ** 0.5)
    qs = 0.5 + _rand((T,), 6).abs()
    b, o = _rand((m,), 7).to(dt), _rand((T, m), 8).to(dt)
    got = pk.linear(q, qs, pk.pack_codes(c, width), scale, bias=b, act=act, other=o, combine=combine, dtype=dt)
    p = (q.double() @ c.double().t()) * scale.double() * qs.double()[:, None]
    z = p + b.double()
    y = _act64(z, act)
    tol = 9 * U32 * (p.abs() + z.abs()) * 1.13 + 8 * U32 * y.abs()
    if combine == "add":
        y = y + o.double()
    else:
        y = y * o.double()
        tol = tol * o.double().abs()
    _inside(got, y, tol + (2 * U32 + _u(dtype)) * y.abs() * 1.01 + _tiny(dtype), "y")


def _mlp(T, d, f, dtype):
    dt, s = _dtype(dtype), d ** -0.5
    return (_rand((T, d), 11).to(dt), _rand((f, d), 12, s).to(dt), _rand((f, d), 13, s).to(dt),
            _rand((T, f), 14, 0.3).to(dt))


def _hidden(x, wg, wu, act):
    d = x.shape[1]
    G, U = x @ wg.t(), x @ wu.t()
    eG = (d + 4) * U32 * (x.abs() @ wg.abs().t())
    eU = (d + 4) * U32 * (x.abs() @ wu.abs().t())
    A, S = _act64(G, act), _slope64(G, act)
    eA = 1.13 * eG + 8 * U32 * (G.abs() + A.abs())
    return U, A, S, eU, eA, eG + 16 * U32 * (1 + G.abs())


@pytest.mark.parametrize("T,d,f", GATED)
@pytest.mark.parametrize("dtype,act", [("bf16", "silu"), ("f16", "gelu")])
def test_gated_mlp_tiles(T, d, f, dtype, act):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp tiles", T, d, f, dtype, act)
    x, wg, wu, _ = _mlp(T, d, f, dtype)
    r = pk.gated_mlp(x, wg, wu, act=act, features=True)
    assert torch.equal(r.h, pk.gated_mlp(x, wg, wu, act=act))
    U, A, S, eU, eA, eS = _hidden(x.double(), wg.double(), wu.double(), act)
    eh = eA * U.abs() + A.abs() * eU + eA * eU + U32 * (A * U).abs()
    _inside(r.h, A * U, eh + _u(dtype) * ((A * U).abs() + eh) + _tiny(dtype), "h")
    _inside(r.up, A, eA, "features of W_up")
    _inside(r.gate, S * U, eS * U.abs() + S.abs() * eU + eS * eU + U32 * (S * U).abs(), "features of W_gate")


@pytest.mark.parametrize("T,d,f,dx,dw", [c[:5] for c in BACKWARD])
@pytest.mark.parametrize("dtype,act", [("bf16", "gelu"), ("f16", "silu")])
def test_gated_mlp_backward_tiles(T, d, f, dx, dw, dtype, act):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp backward tiles", T, d, f, dx, dw, dtype, act)
    x, wg, wu, dh = _mlp(T, d, f, dtype)
    got = pk.gated_mlp_backward(dh, x, wg, wu, act=act, need_dx=dx, need_dw=dw)
    x, wg, wu, dh = x.double(), wg.double(), wu.double(), dh.double()
    U, A, S, eU, eA, eS = _hidden(x, wg, wu, act)
    dG, dU = dh * U * S, dh * A
    u = _u(dtype)
    eDG = dh.abs() * (eU * S.abs() + U.abs() * eS + eU * eS) + 4 * U32 * dG.abs()
    eDG = eDG + u * (dG.abs() + eDG) + _tiny(dtype)
    eDU = dh.abs() * eA + 4 * U32 * dU.abs()
    eDU = eDU + u * (dU.abs() + eDU) + _tiny(dtype)
    aG, aU = dG.abs() + eDG, dU.abs() + eDU

    def check(g, want, err, size, terms, label):
        e = err + (terms + 4) * U32 * size
        _inside(g, want, e + u * (want.abs() + e) + _tiny(dtype), label)
        # entry by entry the bounds add up over the terms; in norm the errors average: 0.6 u of dG, dU and of the
        # result's own rounding each, in squares
        assert float((g.double() - want).norm()) <= (0.85 * u + 1e-5) * float(want.norm()), label
    if dx:
        check(got[0], dG @ wg + dU @ wu, eDG @ wg.abs() + eDU @ wu.abs(), aG @ wg.abs() + aU @ wu.abs(), 2 * f, "dx")
    if dw:
        check(got[1], dG.t() @ x, eDG.t() @ x.abs(), aG.t() @ x.abs(), T, "dw_gate")
        check(got[2], dU.t() @ x, eDU.t() @ x.abs(), aU.t() @ x.abs(), T, "dw_up")
    again = pk.gated_mlp_backward(*(t.to(_dtype(dtype)) for t in (dh, x, wg, wu)), act=act, need_dx=dx, need_dw=dw)
    for a, b in zip(got, again):
        assert a is b is None or torch.equal(a, b)
