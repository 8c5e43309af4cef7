"""GPU tests of the operators around a quantised layer (8-bit norm, product with codes,
gated MLP and its gradients, token log probabilities and their gradients) against
plain implementations in 64 bits on the CPU.

Tolerances are bounds on the roundings that the header allows, in units of
  U32 = 2^-24 (one fp32 rounding), u(dtype) = 2^-24, 2^-11, 2^-8 (the output's).
A sum of n terms in fp32, in any order, is within n U32 of the sum of its terms'
sizes; exp, erf and the like are taken to be within 4 U32.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
NAMES = ("f32", "f16", "bf16")


def _t():
    import torch
    return torch


def _dtype(name):
    torch = _t()
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _u(name):
    return {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[name]


def _tiny(name):   # half the smallest step: what a rounding may lose near zero
    return {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}[name]


def _say(*a):
    print(*a, flush=True)


def _strided(t, pad, shift):
    """The same values in rows `pad` entries longer, `shift` entries off an aligned start."""
    torch = _t()
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), 77, dtype=t.dtype, device=t.device)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def _gen(seed):
    return _t().Generator().manual_seed(seed)


def _rand(shape, seed, scale=1.0):
    return _t().randn(shape, generator=_gen(seed), dtype=_t().float64) * scale


def _within(got, want, tol, label):
    """|got - want| <= tol entrywise; infinities and NaN must be the same."""
    torch = _t()
    got = got.detach().cpu().double()
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), label
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), label
    err = (got - want)[fin].abs()
    lim = torch.broadcast_to(torch.as_tensor(tol, dtype=torch.float64), want.shape)[fin]
    bad = err > lim
    assert not bool(bad.any()), (label, int(bad.sum()), float((err / lim.clamp(min=1e-300)).max()))


# ---------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T,d,residual,weight,pad,shift", [
    (1, 1, False, False, 0, 0), (1, 4096, True, True, 0, 0), (3, 127, True, True, 0, 0),
    (5, 128, False, True, 3, 1), (130, 1000, True, False, 0, 0), (2, 8191, True, True, 1, 3),
    (1030, 520, True, True, 8, 0), (1100, 2049, False, True, 0, 0), (1, 32768, True, True, 0, 0),
    (2, 65536, False, True, 0, 0)])
def test_norm(dtype, T, d, residual, weight, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("norm", dtype, T, d, residual, weight, pad, shift)
    dt = _dtype(dtype)
    x = _rand((T, d), 1).to(dt)
    r = _rand((T, d), 2).to(dt) if residual else None
    w = (1 + 0.1 * _rand((d,), 3)).float() if weight else None
    dev = "cuda:0"
    got = pk.rmsnorm_quant(_strided(x.to(dev), pad, shift), weight=None if w is None else w.to(dev),
                           residual=None if r is None else _strided(r.to(dev), pad, shift), eps=1e-5,
                           with_sum=True, with_y=True)
    torch.cuda.synchronize()
    h = x.double() + (0 if r is None else r.double())
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * (1 if w is None else w.double())
    e = (d + 16) * U32   # relative error of y: the sum of squares, then a few operations
    _within(got.sum, h, U32 * h.abs() + _u(dtype) * h.abs() * (1 + U32) + _tiny(dtype), "sum")
    _within(got.y, y, e * y.abs() + _u(dtype) * y.abs() * (1 + e) + _tiny(dtype), "y")
    scale = y.abs().amax(1) / 127
    _within(got.scale, scale, e * scale, "scale")
    q = got.q.cpu().double()
    _within(q, torch.round(y / scale[:, None]), 1.0, "q")
    # a code is the nearest one, up to the error of y / scale
    assert bool(((q - y / scale[:, None]).abs() <= 0.5 + 127 * 2 * e).all())
    assert int(q.abs().max()) <= 127
    # the padding columns
    full = got.q.as_strided((T, got.q.stride(0) if T > 1 else -(-d // 128) * 128), (got.q.stride(0), 1))
    assert int(full[:, d:].abs().sum()) == 0


@pytest.mark.parametrize("dtype", NAMES)
def test_norm_special_rows(dtype):
    """Rows of zeros, with NaN, with infinity, of tiny numbers; without normalising."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("norm special", dtype)
    dt = _dtype(dtype)
    x = torch.ones((6, 300), dtype=dt)
    x[0] = 0
    x[1, 7] = math.nan
    x[2, 299] = math.inf
    x[3, 0] = -math.inf
    tiny = {"f32": 1e-42, "f16": 6e-8, "bf16": 1e-39}[dtype]
    x[4] = tiny
    for eps in (0.0, 1e-6):
        for normalise in (True, False):
            r = pk.rmsnorm_quant(x.to("cuda:0"), eps=eps, normalise=normalise)
            q, s = r.q.cpu(), r.scale.cpu()
            assert float(s[0]) == 0 and int(q[0].abs().max()) == 0
            for k in (1, 2, 3):
                assert math.isnan(float(s[k])) and int(q[k].abs().max()) == 0, (k, eps, normalise)
            assert bool((q[5] == 127).all())
            if not normalise:
                t = float(x[4, 0].double())
                assert abs(float(s[4]) - t / 127) <= t * 4 * U32 + 2.0 ** -149
    # squares beyond fp32 are not taken for zero
    if dtype != "f16":
        big = torch.full((1, 64), 1e30, dtype=dt, device="cuda:0")
        assert math.isnan(float(pk.rmsnorm_quant(big).scale[0]))


def test_norm_in_place_and_streams():
    """The sum over the residual itself, on a stream of its own."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("norm in place")
    dev = "cuda:0"
    x = _rand((70, 1023), 4).to(dev, torch.bfloat16)
    r = _rand((70, 1023), 5).to(dev, torch.bfloat16)
    want = pk.rmsnorm_quant(x, residual=r)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        keep = r.clone()
        got = pk.rmsnorm_quant(x, residual=keep, sum_out=keep)
    st.synchronize()
    assert got.sum is keep
    for a, b in ((got.q, want.q), (got.scale, want.scale), (keep, want.sum)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- product with codes
def _codes(m, n, width, seed):
    torch = _t()
    top = 8 if width == 4 else 128
    return torch.randint(-top, top, (m, n), generator=_gen(seed), dtype=torch.int8)


def _act64(z, act):
    torch = _t()
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    return z


def _padded_rows(q):
    """q (T x n) in rows padded to a multiple of 128; the padding holds garbage."""
    torch = _t()
    T, n = q.shape
    buf = torch.full((max(T, 1), -(-n // 128) * 128), 99, dtype=torch.int8, device="cuda:0")
    buf[:T, :n] = q.to("cuda:0")
    return buf[:T, :n]


@pytest.mark.parametrize("width", [4, 8])
@pytest.mark.parametrize("n", [1, 5, 127, 128, 129, 1000])
def test_pack_codes(width, n):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("pack", width, n)
    m = 7
    c = _codes(m, n, width, n)
    p = pk.pack_codes(c.to("cuda:0"), width)
    b = p.data.cpu().to(torch.int64)
    np_ = -(-n // 128) * 128
    assert tuple(b.shape) == (m, np_ * width // 8)
    want = torch.zeros((m, np_), dtype=torch.int64)
    want[:, :n] = c
    if width == 8:
        got = torch.where(b > 127, b - 256, b)
    else:
        got = torch.zeros((m, np_), dtype=torch.int64)
        for j in range(np_):
            v = (b[:, j // 8 * 4 + j % 4] >> (4 if j % 8 >= 4 else 0)) & 15
            got[:, j] = torch.where(v > 7, v - 16, v)
    assert torch.equal(got, want)


LINEAR = [
    # T, n, m, width, group, bias, act, combine, dtype
    (1, 1, 1, 4, 0, False, "none", None, "f32"),
    (1, 128, 16, 4, 0, True, "none", None, "bf16"),
    (1, 1000, 333, 4, 64, True, "silu", "add", "bf16"),
    (1, 4096, 1040, 4, 128, False, "none", None, "f16"),
    (2, 257, 65, 8, 0, False, "gelu", "mul", "f32"),
    (7, 640, 100, 8, 128, True, "none", "add", "f16"),
    (16, 4096, 500, 4, 128, True, "silu", "mul", "bf16"),
    (17, 1024, 130, 4, 0, True, "gelu", None, "f32"),
    (33, 777, 257, 4, 192, False, "none", "add", "f32"),
    (64, 512, 64, 8, 64, False, "none", None, "bf16"),
    (130, 300, 1027, 4, 0, True, "silu", "add", "f16"),
    (300, 384, 520, 8, 0, False, "none", "mul", "f32"),
    (513, 1100, 2050, 4, 128, True, "gelu", "add", "bf16"),
    (2050, 200, 2100, 4, 64, False, "none", None, "f32"),
    (4100, 256, 4200, 4, 0, False, "none", "add", "bf16"),
    (4100, 130, 4200, 8, 0, True, "none", None, "f16"),
    # few tiles, a long way to sum
    (70, 3000, 40, 8, 128, True, "gelu", "mul", "f32"),
    (300, 2100, 150, 4, 64, False, "none", None, "bf16"),
    (129, 1500, 33, 4, 0, False, "silu", "add", "f16"),
    # one round of tiles, and more
    (1050, 1100, 2050, 8, 0, True, "none", "add", "bf16"),
    (1050, 900, 2050, 8, 128, False, "silu", None, "f16"),
    (1050, 700, 2050, 8, 64, False, "none", None, "f32"),
    (1050, 1300, 2050, 4, 0, False, "gelu", None, "f16"),
    (2050, 500, 2300, 8, 128, True, "none", None, "bf16"),
    (2050, 500, 2300, 8, 192, False, "none", "mul", "f16"),
]


@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(str(v) for v in c))
def test_linear(case):
    import paper_2608_06291_amd as pk
    torch = _t()
    T, n, m, width, group, bias, act, combine, dtype = case
    _say("linear", case)
    dev, dt = "cuda:0", _dtype(dtype)
    q = torch.randint(-127, 128, (T, n), generator=_gen(1), dtype=torch.int8)
    q[0, 0] = -128
    c = _codes(m, n, width, 2)
    ng = -(-n // group) if group else 1
    scale = (0.01 * (1 + _rand((m, ng) if group else (m,), 3).abs())).float() / math.sqrt(n)
    qs = (0.02 * (1 + _rand((T,), 4).abs())).float()
    b = _rand((m,), 5).to(dt) if bias else None
    o = _rand((T, m), 6).to(dt) if combine else None
    got = pk.linear(_padded_rows(q), qs.to(dev), pk.pack_codes(c.to(dev), width), scale.to(dev),
                    group_size=group, bias=None if b is None else b.to(dev), act=act,
                    other=None if o is None else _strided(o.to(dev), 3, 1), combine=combine, dtype=dt)
    torch.cuda.synchronize()
    parts = torch.zeros((T, m), dtype=torch.float64)
    sizes = torch.zeros((T, m), dtype=torch.float64)
    g = group or n
    for k in range(ng):
        p = q[:, k * g:(k + 1) * g].double() @ c[:, k * g:(k + 1) * g].double().t()
        p = p * (scale[:, k] if group else scale).double()[None, :] * qs.double()[:, None]
        parts += p
        sizes += p.abs()
    z = parts + (0 if b is None else b.double())
    y = _act64(z, act)
    # the sum over groups, three scalings, bias; slope of the activations at most 1.13
    tol = (ng + 8) * U32 * (sizes + z.abs()) * 1.13 + 8 * U32 * y.abs()
    if combine == "add":
        y = y + o.double()
    elif combine == "mul":
        y = y * o.double()
        tol = tol * o.double().abs()
    tol = tol + (2 * U32 + _u(dtype)) * y.abs() * 1.01 + _tiny(dtype)
    _within(got, y, tol, case)


def test_linear_strided_output_repeats_and_in_place():
    """Output rows with gaps, `other` written over, bitwise the same a second time."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear strided")
    dev = "cuda:0"
    T, n, m = 37, 500, 211
    q = torch.randint(-127, 128, (T, n), generator=_gen(1), dtype=torch.int8)
    w = pk.pack_codes(_codes(m, n, 4, 2).to(dev))
    scale = torch.full((m,), 1e-3, device=dev)
    qs = torch.full((T,), 0.5, device=dev)
    o = _rand((T, m), 3).to(dev, torch.bfloat16)
    want = pk.linear(_padded_rows(q), qs, w, scale, other=o)
    buf = torch.full((T, m + 9), 5.0, dtype=torch.bfloat16, device=dev)
    pk.linear(_padded_rows(q), qs, w, scale, other=o, out=buf[:, 4:4 + m])
    assert torch.equal(buf[:, 4:4 + m], want)
    assert bool((buf[:, :4] == 5).all()) and bool((buf[:, 4 + m:] == 5).all())
    pk.linear(_padded_rows(q), qs, w, scale, other=o, out=o)
    assert torch.equal(o, want)
    # T = 0
    assert tuple(pk.linear(_padded_rows(q)[:0], qs[:0], w, scale).shape) == (0, m)


def test_linear_runs_a_solved_layer():
    """From the solver's codes and scales, with the 8-bit rows of the norm."""
    import workloads
    import paper_2608_06291_amd as pk
    torch = _t()
    m, n, T = 130, 200, 19
    _say("linear of a solved layer", m, n)
    p = workloads.make_random(m, n, seed=3)
    A, B, W, s = (torch.from_numpy(p[k]).to("cuda:0") for k in ("A", "B", "W", "scale"))
    f = pk.factor(A, B, p["damp"])
    codes, V = pk.solve(W, f, p["bits"], s)
    f.close()
    x = _rand((T, n), 9).to("cuda:0", torch.bfloat16)
    r = pk.rmsnorm_quant(x)
    y = pk.linear(r.q, r.scale, pk.pack_codes(codes), s, dtype=torch.float32)
    xq = r.q.cpu().double() * r.scale.cpu().double()[:, None]
    want = xq @ V.cpu().double().t()
    size = xq.abs() @ V.cpu().double().abs().t()
    _within(y, want, 8 * U32 * size, "solved")   # V = s * c is rounded once, too


# ---------------------------------------------------------------- gated MLP
def _slope64(z, act):
    torch = _t()
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _mlp64(x, wg, wu, act):
    G, U = x @ wg.t(), x @ wu.t()
    return G, U, _act64(G, act) * U


def _mlp_inputs(T, d, f, dtype, seed):
    dt = _dtype(dtype)
    s = 1.0 / math.sqrt(d)
    return (_rand((T, d), seed).to(dt), _rand((f, d), seed + 1, s).to(dt), _rand((f, d), seed + 2, s).to(dt),
            _rand((T, f), seed + 3, 0.3).to(dt))


def _mlp_errors(x, wg, wu, act):
    """Bounds on the errors of G, U, act(G), act'(G) as computed (slopes at most 1.13, and
    their slopes at most 1)."""
    d = x.shape[1]
    G, U, _ = _mlp64(x, wg, wu, act)
    eG = (d + 4) * U32 * (x.abs() @ wg.abs().t())
    eU = (d + 4) * U32 * (x.abs() @ wu.abs().t())
    eA = 1.13 * eG + 8 * U32 * (G.abs() + _act64(G, act).abs())
    eS = eG + 16 * U32 * (1 + G.abs())
    return G, U, eG, eU, eA, eS


MLP = [(1, 1, 1), (1, 64, 32), (1, 1000, 333), (2, 8, 100), (5, 130, 257), (16, 512, 512), (17, 72, 40),
       (64, 264, 130), (129, 200, 1000), (257, 1000, 270), (700, 96, 1500), (2100, 40, 2200),
       (4100, 40, 2200), (40, 4100, 2200), (4200, 4104, 70),
       # odd rows read a word at a time; whole steps that end with the row
       (3, 97, 33), (30, 1001, 65), (16, 33, 40), (90, 1025, 48), (200, 513, 96),
       # one round of tiles
       (1030, 1100, 1030), (1030, 2050, 300)]


@pytest.mark.parametrize("T,d,f", MLP)
@pytest.mark.parametrize("dtype,act", [("bf16", "silu"), ("f16", "gelu")])
def test_gated_mlp(T, d, f, dtype, act):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp", T, d, f, dtype, act)
    x, wg, wu, _ = _mlp_inputs(T, d, f, dtype, 11)
    pad, shift = ((3, 1) if T % 2 else (8, 0))
    dev = "cuda:0"
    r = pk.gated_mlp(_strided(x.to(dev), pad, shift), wg.to(dev), wu.to(dev), act=act, features=True)
    plain = pk.gated_mlp(x.to(dev), wg.to(dev), wu.to(dev), act=act)
    torch.cuda.synchronize()
    x, wg, wu = x.double(), wg.double(), wu.double()
    G, U, eG, eU, eA, eS = _mlp_errors(x, wg, wu, act)
    A, S = _act64(G, act), _slope64(G, act)
    eh = eA * U.abs() + A.abs() * eU + eA * eU + U32 * (A * U).abs()
    tol = eh + _u(dtype) * ((A * U).abs() + eh) + _tiny(dtype)
    _within(r.h, A * U, tol, "h")
    _within(plain, A * U, tol, "h contiguous")
    _within(r.up, A, eA, "features of W_up")
    _within(r.gate, S * U, eS * U.abs() + S.abs() * eU + eS * eU + U32 * (S * U).abs(), "features of W_gate")


@pytest.mark.parametrize("T,d,f", MLP)
@pytest.mark.parametrize("dtype,act", [("bf16", "gelu"), ("f16", "silu")])
def test_gated_mlp_backward(T, d, f, dtype, act):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp backward", T, d, f, dtype, act)
    x, wg, wu, dh = _mlp_inputs(T, d, f, dtype, 21)
    dev = "cuda:0"
    pad, shift = ((5, 3) if T % 2 else (0, 0))
    dx, dwg, dwu = pk.gated_mlp_backward(_strided(dh.to(dev), pad, shift), _strided(x.to(dev), pad, shift),
                                         wg.to(dev), wu.to(dev), act=act)
    torch.cuda.synchronize()
    x, wg, wu, dh = x.double(), wg.double(), wu.double(), dh.double()
    G, U, eG, eU, eA, eS = _mlp_errors(x, wg, wu, act)
    A, S = _act64(G, act), _slope64(G, act)
    dG, dU = dh * U * S, dh * A
    u = _u(dtype)
    eDG = dh.abs() * (eU * S.abs() + U.abs() * eS + eU * eS) + 4 * U32 * dG.abs()
    eDG = eDG + u * (dG.abs() + eDG) + _tiny(dtype)      # rounded to 16 bits
    eDU = dh.abs() * eA + 4 * U32 * dU.abs()
    eDU = eDU + u * (dU.abs() + eDU) + _tiny(dtype)
    aG, aU = dG.abs() + eDG, dU.abs() + eDU

    def check(got, want, err, size, terms, label):
        e = err + (terms + 4) * U32 * size
        _within(got, want, e + u * (want.abs() + e) + _tiny(dtype), label)
    check(dx, dG @ wg + dU @ wu, eDG @ wg.abs() + eDU @ wu.abs(), aG @ wg.abs() + aU @ wu.abs(), 2 * f, "dx")
    check(dwg, dG.t() @ x, eDG.t() @ x.abs(), aG.t() @ x.abs(), T, "dw_gate")
    check(dwu, dU.t() @ x, eDU.t() @ x.abs(), aU.t() @ x.abs(), T, "dw_up")
    # one of the two alone, the same bits
    only = pk.gated_mlp_backward(dh.to(dev, dx.dtype), x.to(dev, dx.dtype), wg.to(dev, dx.dtype),
                                 wu.to(dev, dx.dtype), act=act, need_dw=False)
    assert only[1] is None and torch.equal(only[0], dx)
    only = pk.gated_mlp_backward(dh.to(dev, dx.dtype), x.to(dev, dx.dtype), wg.to(dev, dx.dtype),
                                 wu.to(dev, dx.dtype), act=act, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dwg) and torch.equal(only[2], dwu)


@pytest.mark.parametrize("T,d,f", [(1, 64, 1), (1, 264, 66), (2, 100, 500), (5, 65, 1024), (33, 72, 70),
                                   (64, 130, 300), (3, 128, 1025), (4, 2048, 1025), (130, 65, 128), (1000, 72, 300)])
@pytest.mark.parametrize("dtype,act", [("bf16", "silu"), ("f16", "gelu")])
def test_gated_mlp_backward_few_tokens(T, d, f, dtype, act):
    """Over few tokens (and features or weights, for dx) or for few weights the gradients are off by no more than their own
    rounding: the norm of the error is that of rounding the 64-bit result, to 5%.  What is
    left of rounding dG and dU is u^2 of them, the fp32 sums and activations a few 1e-6 or
    less; both add in squares to the result's u / 2.5."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp backward, few tokens", T, d, f, dtype, act)
    x, wg, wu, dh = _mlp_inputs(T, d, f, dtype, 91)
    got = pk.gated_mlp_backward(*(t.to("cuda:0") for t in (dh, x, wg, wu)), act=act)
    dt = x.dtype
    x, wg, wu, dh = x.double(), wg.double(), wu.double(), dh.double()
    G, U = x @ wg.t(), x @ wu.t()
    dG, dU = dh * U * _slope64(G, act), dh * _act64(G, act)
    for label, g, want in (("dx", got[0], dG @ wg + dU @ wu), ("dw_gate", got[1], dG.t() @ x),
                           ("dw_up", got[2], dU.t() @ x)):
        if label == "dx" and (T > 64 or (f > 1024 and d * f > 1 << 21)):
            continue
        once = float((want.to(dt).double() - want).norm())
        assert float((g.cpu().double() - want).norm()) <= 1.05 * once + 3e-6 * float(want.norm()), label


@pytest.mark.parametrize("T", [2, 40])
def test_gated_mlp_backward_overflow(T):
    """Gradients of the hidden layer beyond half precision: infinite where they meet one token,
    as without the rests of their rounding."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp backward, overflow", T)
    d, f = 32, 40
    x, wg, wu, dh = (torch.ones(s, dtype=torch.float16, device="cuda:0")
                     for s in ((T, d), (f, d), (f, d), (T, f)))
    x[1:] = 0
    x[1:, 0] = 1
    dh[0, 3] = 60000.0   # dU = 60000 * silu(32), dG = 60000 * 32
    dx, dwg, dwu = pk.gated_mlp_backward(dh, x, wg, wu, act="silu")
    torch.cuda.synchronize()
    assert bool(torch.isposinf(dx[0]).all()) and bool(torch.isfinite(dx[1:]).all())
    for w in (dwg, dwu):
        assert bool(torch.isposinf(w[3]).all())
        rows = torch.arange(f, device="cuda:0") != 3
        assert bool(torch.isfinite(w[rows]).all())


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_mlp_gradient_against_differences(act):
    """The directional derivative of sum(h * dh), from differences of the 64-bit
    forward pass, against the gradients' inner product with the direction.  Central
    differences at 1e-5 are within 1e-8 of the derivative here; the gradients are off
    by at most about 3 u of the sizes summed."""
    import paper_2608_06291_amd as pk
    _say("mlp differences", act)
    T, d, f, dtype = 33, 72, 56, "f16"
    x, wg, wu, dh = _mlp_inputs(T, d, f, dtype, 31)
    grads = [g.cpu().double() for g in pk.gated_mlp_backward(*(t.to("cuda:0") for t in (dh, x, wg, wu)), act=act)]
    base = [t.double() for t in (x, wg, wu)]
    for k in range(3):
        v = _rand(base[k].shape, 41 + k)

        def value(e):
            b = [t + (e * v if i == k else 0) for i, t in enumerate(base)]
            return float((_mlp64(*b, act)[2] * dh.double()).sum())
        diff = (value(1e-5) - value(-1e-5)) / 2e-5
        size = float((grads[k].abs() * v.abs()).sum())
        assert abs(diff - float((grads[k] * v).sum())) <= 3 * _u(dtype) * size + 1e-6, k


@pytest.mark.parametrize("d,ld,shift", [(64, 65, 0), (96, 97, 1), (65, 65, 1), (100, 101, 2), (31, 33, 0)])
def test_gated_mlp_odd_rows(d, ld, shift):
    """Weights and tokens in rows an odd number of entries apart, beginning on a word or off
    one, the last row ending where the buffer ends."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp odd rows", d, ld, shift)
    T, f = 5, 37

    def odd(t):
        rows = t.shape[0]
        buf = torch.full(((rows - 1) * ld + d + shift,), 3.0, dtype=t.dtype, device="cuda:0")
        v = buf[shift:].as_strided((rows, d), (ld, 1))
        v.copy_(t)
        return v
    x, wg, wu, dh = _mlp_inputs(T, d, f, "bf16", 71)
    want = pk.gated_mlp(*(t.to("cuda:0") for t in (x, wg, wu)))
    assert torch.equal(pk.gated_mlp(odd(x), odd(wg), odd(wu)), want)
    a = pk.gated_mlp_backward(*(t.to("cuda:0") for t in (dh, x, wg, wu)))
    b = pk.gated_mlp_backward(dh.to("cuda:0"), odd(x), odd(wg), odd(wu))
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_gated_mlp_no_rows():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp without rows")
    x, wg, wu, dh = (t.to("cuda:0") for t in _mlp_inputs(3, 40, 50, "bf16", 51))
    assert tuple(pk.gated_mlp(x[:0], wg, wu).shape) == (0, 50)
    dx, dwg, dwu = pk.gated_mlp_backward(dh[:0], x[:0], wg, wu)
    torch.cuda.synchronize()
    assert dx.shape[0] == 0 and int(dwg.ne(0).sum()) == 0 and int(dwu.ne(0).sum()) == 0


def test_gated_mlp_non_finite_rows_stay_apart():
    """An infinite or NaN token spoils its own row of h and dx, and no other."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp non-finite")
    x, wg, wu, dh = _mlp_inputs(70, 100, 90, "bf16", 61)
    clean = pk.gated_mlp(x.to("cuda:0"), wg.to("cuda:0"), wu.to("cuda:0"))
    cdx = pk.gated_mlp_backward(*(t.to("cuda:0") for t in (dh, x, wg, wu)), need_dw=False)[0]
    x[3, 99] = math.nan
    x[69, 0] = math.inf
    h = pk.gated_mlp(x.to("cuda:0"), wg.to("cuda:0"), wu.to("cuda:0"))
    dx = pk.gated_mlp_backward(*(t.to("cuda:0") for t in (dh, x, wg, wu)), need_dw=False)[0]
    rows = torch.tensor([r for r in range(70) if r not in (3, 69)], device="cuda:0")
    assert torch.equal(h[rows], clean[rows]) and torch.equal(dx[rows], cdx[rows])
    assert bool(h[3].isnan().all()) and bool(dx[3].isnan().all())


# ---------------------------------------------------------------- token log probabilities
def _logits(T, V, dtype, seed, masked):
    torch = _t()
    z = _rand((T, V), seed, 3.0)
    if masked:
        z[:, 2::5] = -math.inf
        z[T // 2] = -math.inf                      # an empty row
        if T > 3:
            z[1, : V - 1] = -math.inf              # one token left
    return z.to(_dtype(dtype))


def _logprob64(z, target, top):
    torch = _t()
    z = z.double()
    T, V = z.shape
    lse = torch.logsumexp(z, 1)
    empty = lse == -math.inf
    logp = z - torch.where(empty, 0.0, lse)[:, None]
    p = logp.exp()
    H = torch.special.entr(p).sum(1)
    asked = (target >= 0) & (target < V)
    lp = torch.where(asked, logp.gather(1, torch.where(asked, target, 0)[:, None])[:, 0], 0.0)
    order = torch.sort(z, dim=1, descending=True, stable=True)
    idx = order.indices[:, :top]
    return lse, H, lp, idx, logp.gather(1, idx), logp, p


LOGPROB = [(1, 1, 1), (1, 2, 2), (3, 31, 31), (2, 1000, 20), (5, 4096, 1), (1, 8193, 32), (4, 50001, 5),
           (1, 131072, 20), (70, 700, 3), (600, 5001, 8), (3, 200003, 32), (9, 33000, 0)]


def _lp_tolerance(z):
    """Of lse: rounding of the sum (64 terms a thread, then 12 joins and rescalings) and of
    the exponents (up to 100 U32 of each term, most of it from log2 e (z - m))."""
    return 260 * U32


@pytest.mark.parametrize("T,V,top", LOGPROB)
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("masked", [False, True])
def test_token_logprobs(T, V, top, dtype, masked):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob", T, V, top, dtype, masked)
    z = _logits(T, V, dtype, 71, masked)
    target = torch.randint(0, V, (T,), generator=_gen(5))
    if T > 4:
        target[2] = -100
        target[3] = V
    pad, shift = ((1, 3) if V % 2 else (0, 0))
    r = pk.token_logprobs(_strided(z.to("cuda:0"), pad, shift), target.to("cuda:0"), top=top)
    torch.cuda.synchronize()
    lse, H, lp, idx, tlp, _, _ = _logprob64(z, target, top)
    e = _lp_tolerance(z)
    big = 2 * U32 * torch.where(torch.isfinite(lse), lse.abs(), 0.0)
    _within(r.lse, lse, e + big, "lse")
    _within(r.logprob, lp, e + big + 2 * U32 * torch.where(torch.isfinite(lp), lp.abs(), 0.0), "logprob")
    # entropy: the same errors, weighted by |z - m|, at most 60 here
    _within(r.entropy, H, 2 * e * (1 + H) + 8 * U32 * math.log(V + 1), "entropy")
    if top:
        assert torch.equal(r.top_index.cpu(), idx), "top"
        _within(r.top_logprob, tlp, (e + big)[:, None] + 2 * U32 * torch.where(torch.isfinite(tlp), tlp.abs(), 0.0),
                "top logprob")
    # a second call gives the same bits
    again = pk.token_logprobs(_strided(z.to("cuda:0"), pad, shift), target.to("cuda:0"), top=top)
    for a, b in zip(r, again):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("V", [40, 9000, 140000])
def test_token_logprobs_ties(dtype, V):
    """Equal logits (whole rows of them, signed zeros, few values): lowest index first."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob ties", dtype, V)
    z = torch.zeros((4, V), dtype=_dtype(dtype))
    z[1, ::2] = -0.0
    z[2] = torch.randint(0, 3, (V,), generator=_gen(1)).to(z.dtype)
    z[3] = torch.arange(V, 0, -1).clamp(max=V - 7).double().mul(1e-3).to(z.dtype)
    r = pk.token_logprobs(z.to("cuda:0"), None, top=32)
    assert r.logprob is None
    assert torch.equal(r.top_index.cpu(), _logprob64(z, torch.zeros(4, dtype=torch.int64), 32)[3])
    assert abs(float(r.entropy[0]) - math.log(V)) < 1e-4


def test_token_logprobs_uneven_rows():
    """Rows whose large logits sit together, so that a bound from a few places of the row
    is far below the largest ones: rising, falling, one block low."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob uneven")
    V = 32768
    z = torch.rand((5, V), generator=_gen(1)).float()
    z[0] = z[0].sort().values
    z[1] = z[1].sort(descending=True).values
    z[2].view(-1, 4096)[:, :128] -= 50          # what 16 neighbouring threads hold
    z[3].view(-1, 2048)[:, 64:128] -= 50
    z[4, :30000] = -math.inf
    for dt in (torch.float32, torch.float16):
        y = z.to(dt)
        r = pk.token_logprobs(y.to("cuda:0"), None, top=32)
        idx = _logprob64(y, torch.zeros(5, dtype=torch.int64), 32)[3]
        assert torch.equal(r.top_index.cpu(), idx), dt


@pytest.mark.parametrize("V", [300, 70000])
def test_token_logprobs_non_finite(V):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob non-finite", V)
    z = _rand((4, V), 3).float()
    z[0, V - 2] = math.nan
    z[1, 5] = math.inf
    z[2, 7] = 1e30
    r = pk.token_logprobs(z.to("cuda:0"), torch.tensor([1, 5, 7, 3], device="cuda:0"), top=2)
    for k in (0, 1):
        for t in (r.logprob, r.entropy, r.lse):
            assert math.isnan(float(t[k]))
        assert bool(r.top_logprob[k].isnan().all())
    assert int(r.top_index[0, 0]) == V - 2 and int(r.top_index[1, 0]) == 5
    assert float(r.logprob[2]) == 0 and float(r.entropy[2]) == 0 and float(r.lse[2]) == float(z[2, 7])
    assert math.isfinite(float(r.logprob[3]))


@pytest.mark.parametrize("T,V", [(1, 1), (3, 31), (5, 4096), (2, 50001), (70, 700), (300, 9001)])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("masked,entropy", [(False, True), (True, True), (True, False)])
def test_token_logprobs_backward(T, V, dtype, masked, entropy):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob backward", T, V, dtype, masked, entropy)
    z = _logits(T, V, dtype, 81, masked)
    target = torch.randint(0, V, (T,), generator=_gen(6))
    if T > 4:
        target[2] = -1
    gl = _rand((T,), 7).float()
    gh = _rand((T,), 8).float()
    dev = "cuda:0"
    zd = _strided(z.to(dev), 1, 1) if V % 2 else z.to(dev)
    f = pk.token_logprobs(zd, target.to(dev))
    got = pk.token_logprobs_backward(zd, target.to(dev), f.lse, f.entropy if entropy else None, gl.to(dev),
                                     gh.to(dev) if entropy else None)
    torch.cuda.synchronize()
    lse, H, _, _, _, logp, p = _logprob64(z, target, 0)
    alive = (lse > -math.inf)[:, None]
    one = (torch.arange(V)[None] == target[:, None]).double()
    asked = ((target >= 0) & (target < V)).double()[:, None]
    lb = torch.clamp(logp, min=-1e4)
    gl64, gh64 = gl.double()[:, None], gh.double()[:, None] * (1 if entropy else 0)
    want = asked * gl64 * (one - p) - gh64 * p * (lb + H[:, None])
    want = torch.where(alive, want, 0.0)
    # p is off by (error of lse, exponent) of itself; its factor by that of lse and entropy
    ep = _lp_tolerance(z) + 4 * U32 * (1 + lb.abs())
    factor = gl64.abs() + gh64.abs() * (lb.abs() + H[:, None])
    tol = p * factor * ep + p * gh64.abs() * 2 * _lp_tolerance(z) * (2 + H[:, None]) + 4 * U32 * (gl64.abs() * one + p * factor)
    tol = torch.where(alive, tol, 0.0)
    _within(got, want, tol + _u(dtype) * (want.abs() + tol) + _tiny(dtype), "d")
    # over the logits themselves
    same = zd.clone() if zd.is_contiguous() else zd
    pk.token_logprobs_backward(same, target.to(dev), f.lse, f.entropy if entropy else None, gl.to(dev),
                               gh.to(dev) if entropy else None, out=same)
    assert torch.equal(same, got)


def test_token_logprobs_gradient_against_differences():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob differences")
    T, V = 6, 301
    z = _rand((T, V), 91, 2.0).float()
    target = torch.randint(0, V, (T,), generator=_gen(9))
    gl, gh = _rand((T,), 92).float(), _rand((T,), 93).float()
    dev = "cuda:0"
    f = pk.token_logprobs(z.to(dev), target.to(dev))
    d = pk.token_logprobs_backward(z.to(dev), target.to(dev), f.lse, f.entropy, gl.to(dev), gh.to(dev)).cpu().double()
    v = _rand((T, V), 94)

    def value(e):
        y = torch.log_softmax(z.double() + e * v, 1)
        return float((gl.double() * y.gather(1, target[:, None])[:, 0]).sum()
                     - (gh.double() * (y.exp() * y).sum(1)).sum())
    diff = (value(1e-5) - value(-1e-5)) / 2e-5
    # differences: 1e-8; gradients: at most 2 * 260 U32 of the sizes summed
    assert abs(diff - float((d * v).sum())) <= 1e-7 + 600 * U32 * float((d.abs() * v.abs()).sum())


# ---------------------------------------------------------------- offsets beyond 32 bits
def test_logprobs_beyond_32_bits():
    """More than 2^31 logits: the last rows, forward and backward."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob large")
    T, V = 16500, 131072
    z = torch.empty((T, V), dtype=torch.bfloat16, device="cuda:0")
    z.zero_()
    tail = _logits(3, V, "bf16", 131, False)
    z[-3:] = tail.to("cuda:0")
    target = torch.arange(T, dtype=torch.int64)
    r = pk.token_logprobs(z, target.to("cuda:0"), top=3)
    lse, H, lp, idx, _, logp, p = _logprob64(tail, target[-3:], 3)
    _within(r.lse[-3:], lse, 300 * U32 * (1 + lse.abs()), "lse")
    _within(r.logprob[-3:], lp, 300 * U32 * (1 + lp.abs()), "logprob")
    assert torch.equal(r.top_index[-3:].cpu(), idx)
    assert abs(float(r.lse[7]) - math.log(V)) < 1e-4
    pk.token_logprobs_backward(z, target.to("cuda:0"), r.lse, g_logprob=torch.ones(T, device="cuda:0"), out=z)
    one = (torch.arange(V)[None] == target[-3:, None]).double()
    _within(z[-3:], one - p, 2.0 ** -8 * (one - p).abs() + 300 * U32 * (p + one), "d")


def test_linear_beyond_32_bits():
    """More than 2^31 outputs."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear large")
    T, n, m = 66000, 128, 32768
    q = torch.randint(-127, 128, (T, n), generator=_gen(1), dtype=torch.int8)
    c = _codes(m, n, 4, 2)
    y = pk.linear(q.to("cuda:0"), None, pk.pack_codes(c.to("cuda:0")), torch.full((m,), 1e-3, device="cuda:0"))
    for rows in (slice(0, 2), slice(T - 3, T)):
        want = q[rows].double() @ c.double().t() * float(torch.tensor(1e-3, dtype=torch.float32))
        _within(y[rows], want, (2.0 ** -8 + 4 * U32) * want.abs(), "y")


# ---------------------------------------------------------------- refusals of the binding
def test_binding_refuses_what_does_not_fit():
    import paper_2608_06291_amd as pk
    torch = _t()
    dev = "cuda:0"
    bf = dict(dtype=torch.bfloat16, device=dev)
    x, w = torch.zeros((4, 64), **bf), torch.zeros((8, 64), **bf)
    with pytest.raises(ValueError):
        pk.gated_mlp(x, w, w[:4])
    with pytest.raises(ValueError):
        pk.gated_mlp(x, w[:, :32], w[:, :32])
    with pytest.raises(TypeError):
        pk.gated_mlp(x, w.float(), w)
    with pytest.raises(ValueError):
        pk.gated_mlp(x.t(), w, w)
    with pytest.raises(pk.BakronError):
        pk.gated_mlp(x.float(), w.float(), w.float())
    with pytest.raises(KeyError):
        pk.gated_mlp(x, w, w, act="tanh")
    with pytest.raises(ValueError):
        pk.gated_mlp(x[:1].expand(4, 64), w, w)               # rows that overlap
    with pytest.raises(ValueError):
        pk.gated_mlp_backward(x, x, w, w)
    q = torch.zeros((4, 100), dtype=torch.int8, device=dev)    # rows that are not padded
    codes = pk.pack_codes(torch.zeros((8, 100), dtype=torch.int8, device=dev))
    with pytest.raises((ValueError, pk.BakronError)):
        pk.linear(q, None, codes, torch.ones(8, device=dev))
    good = _padded_rows(q.cpu())
    with pytest.raises(ValueError):
        pk.linear(good, None, codes, torch.ones(9, device=dev))
    with pytest.raises(ValueError):
        pk.linear(good, torch.ones(5, device=dev), codes, torch.ones(8, device=dev))
    with pytest.raises(TypeError):
        pk.linear(good.float(), None, codes, torch.ones(8, device=dev))
    with pytest.raises(pk.BakronError):
        pk.linear(good, None, codes, torch.ones((8, 4), device=dev), group_size=32)
    with pytest.raises(ValueError):
        pk.linear(good, None, codes, torch.ones(8, device=dev), other=torch.zeros((4, 7), **bf))
    z = torch.zeros((4, 50), device=dev)
    with pytest.raises(TypeError):
        pk.token_logprobs(z, torch.zeros(4, dtype=torch.int32, device=dev))
    with pytest.raises(pk.BakronError):
        pk.token_logprobs(z, None, top=51)
    with pytest.raises(TypeError):
        pk.token_logprobs(z.double())
    with pytest.raises(ValueError):
        pk.rmsnorm_quant(x, weight=torch.ones(63, device=dev))
    with pytest.raises(pk.BakronError):
        pk.rmsnorm_quant(x, eps=-1.0)


# ---------------------------------------------------------------- capture into graphs
def test_operators_replay_from_a_graph():
    """All operators in one graph, replayed three times on changed inputs with eager
    work in between: every replay gives the eager results, bit for bit."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("graph")
    dev = "cuda:0"
    T, d, f, V = 9, 264, 136, 9000
    x, wg, wu, dh = (t.to(dev) for t in _mlp_inputs(T, d, f, "bf16", 101))
    w = pk.pack_codes(_codes(d, f, 4, 3).to(dev))
    s = torch.full((d,), 1e-2, device=dev)
    z = _logits(T, V, "bf16", 102, True).to(dev)
    target = torch.randint(0, V, (T,), generator=_gen(1)).to(dev)
    gl = torch.ones(T, device=dev)

    def step():
        n = pk.rmsnorm_quant(x, residual=x, with_y=True)
        h = pk.gated_mlp(n.y, wg, wu)
        q = pk.rmsnorm_quant(h, normalise=False)
        y = pk.linear(q.q, q.scale, w, s, other=n.sum)
        g = pk.gated_mlp_backward(dh, n.y, wg, wu)
        lp = pk.token_logprobs(z, target, top=5)
        dz = pk.token_logprobs_backward(z, target, lp.lse, lp.entropy, gl, gl)
        return [n.q.contiguous(), n.scale, n.sum, h, y, *g, *lp, dz]

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for k in range(3):
        x.copy_(_rand((T, d), 110 + k).to(torch.bfloat16))
        z.copy_(_logits(T, V, "bf16", 120 + k, True))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), (k, i)
