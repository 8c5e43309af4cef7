"""GPU tests of the operators around a quantised layer where numbers leave the middle of
their range: the smallest and largest ones, a common offset, the tails of the activations.

Tolerances as in test_gpu_operators.py: bounds on the roundings that the header allows.
"""
import math

import pytest

from test_gpu_operators import U32, _act64, _dtype, _gen, _rand, _say, _slope64, _t, _tiny, _u, _within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ---------------------------------------------------------------- norm
def test_norm_codes_of_subnormal_rows():
    """Rows whose largest value is 1 to 16000 steps of the smallest fp32 number: scale = top / 127 is then a
    few steps itself, rounded by up to a half of one, and value / scale leaves [-127, 127]."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("norm subnormal codes")
    tops = torch.cat((torch.arange(1, 2000), torch.arange(2000, 16001, 7)))
    steps = torch.stack((tops, -tops, tops // 2, torch.zeros_like(tops), -(tops // 3)), 1).double()
    x = (steps * 2.0 ** -149).float()
    assert torch.equal(x.double(), steps * 2.0 ** -149)
    r = pk.rmsnorm_quant(x.to(DEV), normalise=False)
    q, s = r.q.cpu().double(), r.scale.cpu().double()
    # the scale is the nearest number of steps to top / 127
    assert bool(((s * 2.0 ** 149 - tops / 127).abs() <= 0.5).all())
    zero = s == 0
    assert int(q[zero].abs().sum()) == 0
    want = (x.double() / torch.where(zero, 1.0, s)[:, None]).clamp(-127, 127)
    err = torch.where(zero[:, None], 0.0, q - want).abs()
    assert bool((err <= 0.5 + 127 * 4 * U32).all()), float(err.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 1003, 20000])
def test_norm_of_tiny_rows_without_eps(dtype, d):
    """eps = 0: the mean of squares of rows down to the smallest numbers is not lost."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("norm tiny", dtype, d)
    x = _rand((12, d), 3).clamp(-4, 4) * 2.0 ** torch.tensor([-10, -55, -59, -60, -61, -62, -63, -70, -75, -90, -110, -130])[:, None]
    x = x.to(_dtype(dtype))
    for w in (None, (1 + 0.1 * _rand((d,), 4)).float()):
        r = pk.rmsnorm_quant(x.to(DEV), weight=None if w is None else w.to(DEV), eps=0.0, with_y=True)
        h = x.double()
        y = h / torch.sqrt((h * h).mean(1, keepdim=True)) * (1 if w is None else w.double())
        # squares that are subnormal beside a mean of 2^-120 or more: a step of 2^-149 each
        e = (d + 16) * U32 + 2.0 ** -29
        _within(r.y, y, e * y.abs() + _u(dtype) * y.abs() * (1 + e) + _tiny(dtype), "y")
        _within(r.scale, y.abs().amax(1) / 127, e * y.abs().amax(1) / 127, "scale")


# ---------------------------------------------------------------- gated MLP, gradients in half precision
def _backward_check(x, wg, wu, dh, act, want_dx=True, want_dw=True):
    """Half-precision gradients against 64 bits.  Of dG and dU, what is kept is the nearest 11-bit number, and
    of small ones no less than 2^-39 of the largest of all (11 bits of 2^15 go down to 2^-24; half a step)
    or 2^-25, whichever is more where the largest is 1 or more."""
    import paper_2608_06291_amd as pk
    torch = _t()
    T, d = x.shape
    f = wg.shape[0]
    got = pk.gated_mlp_backward(*(t.to(DEV) for t in (dh, x, wg, wu)), act=act)
    torch.cuda.synchronize()
    x, wg, wu, dh = x.double(), wg.double(), wu.double(), dh.double()
    G, U = x @ wg.t(), x @ wu.t()
    eG = (d + 4) * U32 * (x.abs() @ wg.abs().t())
    eU = (d + 4) * U32 * (x.abs() @ wu.abs().t())
    A, S = _act64(G, act), _slope64(G, act)
    eA = 1.13 * eG + 8 * U32 * (G.abs() + A.abs())
    eS = eG + 16 * U32 * (1 + G.abs())
    dG, dU = dh * U * S, dh * A
    most = float(max(dG.abs().max(), dU.abs().max()))
    lost = 2.0 ** -39 * most if most < 1 or most > 2.0 ** 15 else 2.0 ** -25
    u = _u("f16")
    eDG = dh.abs() * (eU * S.abs() + U.abs() * eS + eU * eS) + 4 * U32 * dG.abs()
    eDG = eDG + u * (dG.abs() + eDG) + lost
    eDU = dh.abs() * eA + 4 * U32 * dU.abs()
    eDU = eDU + u * (dU.abs() + eDU) + lost

    def check(g, want, err, size, terms, label):
        e = err + (terms + 4) * U32 * size
        e = e + u * (want.abs() + e) + _tiny("f16")
        far = want.abs() > 65520 + e             # rounds to infinity
        near = (want.abs() > 65504 - e) & ~far   # may or may not
        g = g.cpu().double()
        assert bool((g[far] == torch.sign(want[far]) * math.inf).all()), label
        err = torch.where(far | near, 0.0, (g - want).abs())
        assert bool((err <= e).all()), (label, float((err / e).max()))   # (NaN fails, too)
    aG, aU = dG.abs() + eDG, dU.abs() + eDU
    if want_dx:
        check(got[0], dG @ wg + dU @ wu, eDG @ wg.abs() + eDU @ wu.abs(), aG @ wg.abs() + aU @ wu.abs(), 2 * f, "dx")
    if want_dw:
        check(got[1], dG.t() @ x, eDG.t() @ x.abs(), aG.t() @ x.abs(), T, "dw_gate")
        check(got[2], dU.t() @ x, eDU.t() @ x.abs(), aU.t() @ x.abs(), T, "dw_up")
    return got, (dG, dU, x, wg, wu)


def _half_inputs(T, d, f, size, seed=21):
    s = 1.0 / math.sqrt(d)
    return (_rand((T, d), seed).half(), _rand((f, d), seed + 1, s).half(), _rand((f, d), seed + 2, s).half(),
            _rand((T, f), seed + 3, size).half())


@pytest.mark.parametrize("T,d,f", [(256, 512, 1376), (5, 96, 130), (40, 333, 70), (1500, 264, 2100)])
@pytest.mark.parametrize("size", [1e-3, 1e-5, 3e-7])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_half_gradients_of_small_losses(T, d, f, size, act):
    """dh as a loss that is a mean over many tokens has it, without a scale of its own."""
    _say("half gradients, small", T, d, f, size, act)
    torch = _t()
    x, wg, wu, dh = _half_inputs(T, d, f, size)
    got, (dG, dU, x, wg, wu) = _backward_check(x, wg, wu, dh, act)
    # in norm: the rounding of dG and dU (each entry within u, 0.6 u at most in the mean square) and the result's own
    # beside it; 1e-5 for fp32 sums
    for g, want in ((got[0], dG @ wg + dU @ wu), (got[1], dG.t() @ x), (got[2], dU.t() @ x)):
        once = (want.half().double() - want).norm()
        assert float((g.cpu().double() - want).norm()) <= 1.05 * float(once) + (0.6 * _u("f16") + 1e-5) * float(want.norm())


@pytest.mark.parametrize("T,d,f", [(200, 330, 500), (7, 96, 64)])
def test_half_gradients_beyond_the_largest_number(T, d, f):
    """dG beyond 65504 where small weights bring dx back into range."""
    _say("half gradients, large", T, d, f)
    torch = _t()
    s = 1.0 / math.sqrt(d)
    x, wu = _rand((T, d), 1, 4.0).half(), _rand((f, d), 2, s).half()
    wg = _rand((f, d), 3, 1e-3 * s).half()
    dh = (_rand((T, f), 4).sign() * 6e4).half()
    got, _ = _backward_check(x, wg, wu, dh, "silu")
    assert bool(torch.isfinite(got[0]).all()) and bool(torch.isfinite(got[2]).all())


def test_half_gradients_spoiled_and_empty():
    """NaN and infinities in dh spoil what they meet, and do not set the scale of the rest; all zeros give zeros."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("half gradients, spoiled")
    x, wg, wu, dh = (t.to(DEV) for t in _half_inputs(70, 100, 90, 1e-5))
    clean = pk.gated_mlp_backward(dh, x, wg, wu, need_dw=False)[0]
    bad = dh.clone()
    bad[3, 5], bad[69, 0] = math.nan, math.inf
    got = pk.gated_mlp_backward(bad, x, wg, wu, need_dw=False)[0]
    rows = torch.tensor([r for r in range(70) if r not in (3, 69)], device=DEV)
    assert torch.equal(got[rows], clean[rows])
    assert bool(got[3].isnan().all()) and not bool(got[69].isfinite().any())
    for g in pk.gated_mlp_backward(torch.zeros_like(dh), x, wg, wu):
        assert int(g.ne(0).sum()) == 0


def test_half_gradients_replay_from_a_graph():
    """One graph over inputs that need the second run, and do not, and need it again."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("half gradients, graph")
    for T, d, f in ((9, 264, 136), (700, 264, 1000)):
        x, wg, wu, _ = (t.to(DEV) for t in _half_inputs(T, d, f, 1.0))
        dh = torch.zeros((T, f), dtype=torch.float16, device=DEV)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            pk.gated_mlp_backward(dh, x, wg, wu)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = pk.gated_mlp_backward(dh, x, wg, wu)
        for k, size in enumerate((1e-5, 0.3, 1e-6, 2e4)):
            dh.copy_((_rand((T, f), 30 + k) * size).half())
            want = [t.clone() for t in pk.gated_mlp_backward(dh, x, wg, wu)]
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and int(a.ne(0).sum()) > 0, (k, T)   # (NaN, too)


# ---------------------------------------------------------------- log probabilities
@pytest.mark.parametrize("T,V,top", [(3, 1000, 5), (2, 60000, 20), (1, 131072, 1), (300, 5001, 3)])
@pytest.mark.parametrize("offset", [1e3, -1e4])
def test_token_logprobs_with_an_offset(T, V, top, offset):
    """A constant added to a row changes nothing: log probabilities are as good as without it."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob offset", T, V, top, offset)
    z = (_rand((T, V), 5, 3.0) + offset).float()
    # likely and unlikely targets
    target = torch.where(torch.arange(T) % 3 > 0, z.argmax(1), torch.arange(T) % V)
    z[torch.arange(T), target] += 10.0 * (torch.arange(T) % 2)
    r = pk.token_logprobs(z.to(DEV), target.to(DEV), top=top)
    zd = z.double()
    m = zd.amax(1, keepdim=True)
    logp = (zd - m) - (zd - m).exp().sum(1, keepdim=True).log()
    lp = logp.gather(1, target[:, None])[:, 0]
    # log of the sum: see _lp_tolerance; z - m is exact or rounded once
    e = 260 * U32
    _within(r.logprob, lp, e + 3 * U32 * lp.abs(), "logprob")
    best = torch.sort(zd, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(r.top_index.cpu(), best)
    t = logp.gather(1, best)
    _within(r.top_logprob, t, e + 3 * U32 * t.abs(), "top")


def test_token_logprobs_gradient_of_unlikely_tokens():
    """p of unlikely tokens in fp32, to the rounding of z - lse and a few more."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("logprob gradient, unlikely")
    V = 4000
    z = (-torch.rand((3, V), generator=_gen(1), dtype=torch.float64) * 80).float()
    z[:, 0] = 0
    lse = torch.logsumexp(z.double(), 1).float()
    d = pk.token_logprobs_backward(z.to(DEV), torch.zeros(3, dtype=torch.int64, device=DEV), lse.to(DEV),
                                   g_logprob=torch.full((3,), -1.0, device=DEV))
    lp = z.double() - lse.double()[:, None]
    p = lp.exp()
    # z - lse rounded once (an error of the exponent, so relative in p), exp2 and its argument 4 units
    tol = p * (U32 * lp.abs() * 1.01 + 4 * U32)
    _within(d[:, 1:], p[:, 1:], tol[:, 1:], "p")


# ---------------------------------------------------------------- activations
def _activation_through_linear(z, act):
    """act(z) in fp32 by a product whose sums are exact: z (n) multiples of 1/64 below 250 in size."""
    import paper_2608_06291_amd as pk
    torch = _t()
    k = (z * 64).round().to(torch.int64)
    n, T = 256, z.numel()
    q = torch.zeros((T, n), dtype=torch.int8)
    left = k.clone()
    for j in range(127):   # k as a sum of entries of at most 127
        step = left.clamp(-127, 127)
        q[:, j] = step.to(torch.int8)
        left -= step
    assert int(left.abs().sum()) == 0
    codes = torch.ones((16, n), dtype=torch.int8, device=DEV)
    y = pk.linear(q.to(DEV), None, pk.pack_codes(codes, 8), torch.full((16,), 1.0 / 64, device=DEV), act=act,
                  dtype=torch.float32)
    assert bool((y == y[:, :1]).all())
    return y[:, 0]


def test_silu_of_negative_numbers():
    torch = _t()
    _say("silu tail")
    z = torch.arange(-85 * 64, 60 * 64, dtype=torch.float64) / 64
    want = z * torch.sigmoid(z)
    # exp2 of a two-part argument, sum, reciprocal, product: a unit or two each
    _within(_activation_through_linear(z, "silu"), want, 8 * U32 * want.abs(), "silu")


def test_gelu_of_negative_numbers():
    torch = _t()
    _say("gelu tail")
    z = torch.arange(-12 * 64, 12 * 64, dtype=torch.float64) / 64
    want = z * 0.5 * torch.special.erfc(-z * math.sqrt(0.5))   # (ndtr is 1 + erf: nothing is left of it at -9)
    # a polynomial within 2e-7 relative to the tail, exp2 of a two-part argument, products
    _within(_activation_through_linear(z, "gelu"), want, (2e-7 + 10 * U32) * want.abs(), "gelu")


# ---------------------------------------------------------------- order of sums
@pytest.mark.parametrize("T", [1, 5, 16, 17, 30])
@pytest.mark.parametrize("d", [129, 257, 513, 1001, 2049])
def test_gated_mlp_sums_do_not_depend_on_alignment(T, d):
    """The same values in rows an odd and an even number of entries apart: the same bits."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp order", T, d)
    f = 70
    x, wg, wu, dh = _half_inputs(T, d, f, 0.3, seed=5)

    def rows(t, ld):
        buf = torch.zeros((t.shape[0], ld), dtype=t.dtype, device=DEV)
        buf[:, :d] = t.to(DEV)
        return buf[:, :d]
    a, b = ([rows(t, ld) for t in (x, wg, wu)] for ld in (d | 1, (d + 8) // 8 * 8))
    assert a[0].stride(0) % 2 == 1 or T == 1
    assert torch.equal(pk.gated_mlp(*a), pk.gated_mlp(*b))
    for p, q in zip(pk.gated_mlp_backward(dh.to(DEV), *a), pk.gated_mlp_backward(dh.to(DEV), *b)):
        assert torch.equal(p, q)
