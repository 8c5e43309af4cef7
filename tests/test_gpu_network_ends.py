"""GPU tests of the operators at the two ends of a network and of its norms (vocabulary loss without
logits, layer norm, embedding; each with its gradient) against plain implementations in 64 bits on
the CPU.

Tolerances are bounds on the roundings that the header allows, in units of U32 = 2^-24 (one fp32 rounding)
and u(dtype) = 2^-24, 2^-11, 2^-8 (the output's).  A sum of n terms in fp32, in any order, is within n U32
of the sum of its terms' sizes; exp, log and the like are taken to be within 4 U32.
"""
import math

import pytest

from network_ends_sizes import HEAD, HEAD_LARGE

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
NAMES = ("f32", "f16", "bf16")
DEV = "cuda:0"


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
    """The same values on the GPU in rows `pad` entries longer, `shift` entries off an aligned start."""
    torch = _t()
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 8,), 77, dtype=t.dtype, device=DEV)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def _rand(shape, seed, scale=1.0):
    torch = _t()
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale


def _within(got, want, tol, label):
    """|got - want| <= tol entrywise; infinities and NaN must be the same."""
    torch = _t()
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (label, got.shape, want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), label
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), label
    err = (got - want)[fin].abs()
    lim = torch.broadcast_to(torch.as_tensor(tol, dtype=torch.float64), want.shape)[fin]
    bad = err > lim
    assert not bool(bad.any()), (label, int(bad.sum()), float((err / lim.clamp(min=1e-300)).max()))


# ---------------------------------------------------------------- embedding
EMBED = [(1, 1, 1, 0, 0), (1, 4096, 1000, 0, 0), (5, 7, 3, 0, 0), (200, 127, 50, 3, 1), (1000, 520, 90, 8, 0),
         (3000, 64, 20000, 0, 0), (130, 8193, 33, 1, 3), (4097, 96, 2, 0, 0), (70, 1028, 5, 0, 0),
         (256, 40, 2000, 0, 0), (257, 40, 2000, 0, 0), (255, 640, 7, 0, 0), (300, 1100, 11, 0, 0), (65, 3, 5000, 0, 0)]


def _tokens(T, V, seed):
    torch = _t()
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g)
    if T > 3:
        t[::7] = V // 2                       # one frequent token
        t[1::11] = -100
        t[2::13] = V                          # the first one outside
        t[3::17] = (1 << 40) + 1              # .. and one that a 32-bit number would take for 1
    return t


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T,d,V,pad,shift", EMBED)
def test_embedding(dtype, T, d, V, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("embedding", dtype, T, d, V, pad, shift)
    dt = _dtype(dtype)
    table, tok, scale = _rand((V, d), 1).to(dt), _tokens(T, V, 2), 1.7
    got = pk.embedding(tok.to(DEV), _strided(table, pad, shift), scale=scale)
    torch.cuda.synchronize()
    asked = (tok >= 0) & (tok < V)
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    want = torch.where(asked[:, None], table.double()[tok.clamp(0, V - 1)] * s32, 0.0)
    _within(got, want, (U32 + _u(dtype) * (1 + U32)) * want.abs() + _tiny(dtype), "rows")
    assert torch.equal(pk.embedding(tok.to(DEV), table.to(DEV)).cpu(),
                       torch.where(asked[:, None], table[tok.clamp(0, V - 1)], torch.zeros((), dtype=dt)))


def _embed_grad(dy, tok, V, scale):
    """(sum, sum of sizes, terms) of each row."""
    torch = _t()
    asked = (tok >= 0) & (tok < V)
    k = tok[asked]
    out, size = (torch.zeros((V, dy.shape[1]), dtype=torch.float64).index_add_(0, k, f(dy[asked].double()) * scale)
                 for f in (lambda v: v, torch.abs))
    return out, size, torch.bincount(k, minlength=V)[:, None]


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T,d,V,pad,shift", EMBED)
def test_embedding_backward(dtype, T, d, V, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("embedding backward", dtype, T, d, V, pad, shift)
    dt, scale = _dtype(dtype), 0.75
    dy, tok = _rand((T, d), 1).to(dt), _tokens(T, V, 2)
    sums, size, n = _embed_grad(dy, tok, V, scale)
    tol = (n + 2) * U32 * size
    x = _strided(dy, pad, shift)
    got = pk.embedding_backward(x, tok.to(DEV), V, scale=scale)
    _within(got, sums, tol + _u(dtype) * (sums.abs() + tol) + _tiny(dtype), "gradient")
    # on top of another gradient, out of place and in place
    base = _rand((V, d), 3).to(dt)
    want = sums + base.double()
    lim = tol + U32 * want.abs()
    lim = lim + _u(dtype) * (want.abs() + lim) + _tiny(dtype)
    b = _strided(base, pad, shift)
    got = pk.embedding_backward(x, tok.to(DEV), V, scale=scale, base=b)
    _within(got, want, lim, "with a base")
    assert torch.equal(b.cpu(), base)
    again = pk.embedding_backward(x, tok.to(DEV), V, scale=scale, base=b, out=b)
    assert torch.equal(again, got) and again.data_ptr() == b.data_ptr()
    # rows of nothing
    none = torch.full((T,), -1, device=DEV)
    assert not bool(pk.embedding_backward(x, none, V).any())
    assert torch.equal(pk.embedding_backward(x, none, V, base=base.to(DEV)).cpu(), base)
    assert torch.equal(pk.embedding_backward(x[:0], none[:0], V, base=base.to(DEV)).cpu(), base)


@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("d,V,pad,shift", [(1, 70, 0, 1), (7, 70, 1, 0), (33, 90, 0, 3), (63, 90, 2, 1), (17, 50, 0, 1), (64, 40, 8, 0), (64, 40, 1, 1), (201, 60, 0, 5),
                                           (2051, 25, 4, 2), (4100, 19, 0, 0), (4100, 17000, 12, 8), (4096, 17000, 16, 16)])
def test_embedding_backward_into_rows(dtype, T, d, V, pad, shift):
    """The gradient in rows of a wider buffer at any alignment: rows of no token are zeros, nothing else is written."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("embedding backward into rows", dtype, T, d, V, pad, shift)
    dt = _dtype(dtype)
    dy, tok = _rand((T, d), 1).to(dt).to(DEV), _tokens(T, V, 2).clamp(max=V // 2).to(DEV)   # (half of the rows without one)
    want = pk.embedding_backward(dy, tok, V, base=torch.zeros(V, d, dtype=dt, device=DEV))
    buf = torch.full((shift + V * (d + pad) + 64,), 9.0, dtype=dt, device=DEV)
    out = buf[shift:shift + V * (d + pad)].view(V, d + pad)
    pk.embedding_backward(dy, tok, V, out=out[:, :d])
    assert torch.equal(out[:, :d], want) and not bool(out[V // 2 + 1:, :d].any())
    assert bool((buf[:shift] == 9).all()) and bool((buf[shift + V * (d + pad):] == 9).all()) and bool((out[:, d:] == 9).all())


# ---------------------------------------------------------------- layer norm
NORM = [(1, 1, False, 0, 0), (1, 4096, True, 0, 0), (3, 127, True, 0, 0), (5, 128, False, 3, 1), (130, 1000, True, 0, 0),
        (2, 8191, True, 1, 3), (1030, 520, True, 8, 0), (1100, 2049, False, 0, 0), (1, 32768, True, 0, 0),
        (2, 65536, False, 0, 0), (257, 7, True, 0, 0), (40, 16384, True, 0, 0),
        (32, 1001, True, 0, 0), (33, 1001, True, 0, 0), (31, 70, True, 3, 1)]


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T,d,residual,pad,shift", NORM)
def test_layernorm(dtype, centre, T, d, residual, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("layernorm", dtype, centre, T, d, residual, pad, shift)
    dt, eps = _dtype(dtype), 1e-5
    x = (_rand((T, d), 1) + 3.0).to(dt)
    r = _rand((T, d), 2).to(dt) if residual else None
    w, b = (1 + 0.1 * _rand((d,), 3)).float(), (0.1 * _rand((d,), 4)).float()
    for weight, bias in ((w, b), (None, None)):
        got = pk.layernorm(_strided(x, pad, shift), None if weight is None else weight.to(DEV),
                           None if bias is None else bias.to(DEV),
                           residual=None if r is None else _strided(r, pad, shift), eps=eps, centre=centre)
        torch.cuda.synchronize()
        h = x.double()
        if residual:
            h = h + r.double()
            _within(got.sum, h, U32 * h.abs() + _u(dtype) * h.abs() * (1 + U32) + _tiny(dtype), "sum")
            h = got.sum.cpu().double()   # the norm is that of the rounded stream
        else:
            assert got.sum is None
        mean = h.mean(1, keepdim=True) if centre else torch.zeros((T, 1), dtype=torch.float64)
        # eps is passed in 32 bits; where a row's deviation is 0 (one entry), it is all there is
        e32 = float(torch.tensor(eps, dtype=torch.float32))
        var = (h - mean).square().mean(1, keepdim=True)
        rstd = 1 / torch.sqrt(var + e32)
        # mean: d roundings of sums and one of the result.  Off from it by that much, the entries lose a rounding
        # of their own each (h - mean); their sum, d roundings more, is taken off.  Entry: n is off by the roundings of
        # h - mean, of the rest's and of rstd's.
        top = h.abs().amax(1, keepdim=True)
        if centre:
            _within(got.mean, mean[:, 0], ((d + 2) * U32 * h.abs().mean(1) + U32 * mean[:, 0].abs()), "mean")
        else:
            assert got.mean is None
        dev = (h - mean).abs()
        off = (d + 4) * U32 * ((h - mean).abs().mean(1, keepdim=True) + (d + 2) * U32 * top) if centre else 0 * top
        off = off + (U32 * (dev + (d + 2) * U32 * top) if centre else 0.0)      # absolute error of h - mean
        # relative error of var + eps: its sum, and the entries' errors (their own roundings and the mean's square)
        evar = (d + 6) * U32 + 2 * (off.amax(1, keepdim=True) * dev.mean(1, keepdim=True)) / (var + e32) + \
            (off.amax(1, keepdim=True) ** 2) / (var + e32) if centre else (d + 6) * U32
        er = evar + 4 * U32
        _within(got.rstd, rstd[:, 0], (er * rstd)[:, 0], "rstd")
        wd = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
        bd = torch.zeros(d, dtype=torch.float64) if bias is None else bias.double()
        n = (h - mean) * rstd
        y = wd * n + bd
        en = (n.abs() * (er + 4 * U32) + off * rstd * (1 + er)) * wd.abs()
        e = en + 2 * U32 * (y.abs() + (wd * n).abs())
        _within(got.y, y, e + _u(dtype) * (y.abs() + e) + _tiny(dtype), "y")


@pytest.mark.parametrize("dtype", NAMES)
def test_layernorm_special_rows(dtype):
    """Rows of zeros, of one value, far from zero, with NaN or infinities."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("layernorm special", dtype)
    dt = _dtype(dtype)
    x = _rand((8, 300), 5).to(dt)
    x[0] = 0
    x[1, 7] = math.nan
    x[2, 299] = math.inf
    x[3, 0] = -math.inf
    x[4] = 3
    x[5] = (x[5].double() * 1e-3 + 2048 / 32).to(dt)
    bias = torch.full((300,), 0.5, device=DEV)
    for centre in (True, False):
        g = pk.layernorm(x.to(DEV), bias=bias, centre=centre)
        y, r = g.y.cpu(), g.rstd.cpu()
        for k in (1, 2, 3):
            assert bool(torch.isnan(y[k]).all()) and math.isnan(float(r[k])), (k, centre)
        assert bool((y[0] == 0.5).all()) and abs(float(r[0]) - 1e-5 ** -0.5) < 1e-4 * 1e-5 ** -0.5
        if centre:
            assert bool((y[4] == 0.5).all()) and float(g.mean[4]) == 3
        for k in (6, 7):   # the rows beside them as if alone
            one = pk.layernorm(x[k:k + 1].to(DEV), bias=bias, centre=centre)
            assert torch.equal(one.y[0].cpu(), y[k])
    if dtype != "f16":   # squares beyond fp32 are not taken for zero
        big = torch.full((1, 64), 1e30, dtype=dt, device=DEV)
        assert math.isnan(float(pk.layernorm(big, centre=False).rstd[0]))


def _norm_grad(x, dy, w, mean, rstd, ds, centre):
    n = (x - mean) * rstd
    g = dy * w
    mg, mn = g.mean(1, keepdim=True) if centre else 0 * mean, (g * n).mean(1, keepdim=True)
    dx = rstd * (g - mg - n * mn) + ds
    return dx, (dy * n).sum(0), dy.sum(0), n, g, mg, mn


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("dtype", NAMES)
@pytest.mark.parametrize("T,d,residual,pad,shift", NORM + [(4000, 256, True, 0, 0)])
def test_layernorm_backward(dtype, centre, T, d, residual, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("layernorm backward", dtype, centre, T, d, residual, pad, shift)
    dt = _dtype(dtype)
    x, dy = (_rand((T, d), 1) + 0.5).to(dt), _rand((T, d), 2).to(dt)
    ds = _rand((T, d), 3).to(dt) if residual else None
    w = (1 + 0.1 * _rand((d,), 4)).float()
    f = pk.layernorm(x.to(DEV), w.to(DEV), centre=centre)
    mean = f.mean.cpu().double()[:, None] if centre else torch.zeros((T, 1), dtype=torch.float64)
    rstd = f.rstd.cpu().double()[:, None]
    xs, gs = _strided(x, pad, shift), _strided(dy, pad, shift)
    args = (gs, xs, w.to(DEV), f.mean, f.rstd)
    dx, dw, db = pk.layernorm_backward(*args, d_sum=None if ds is None else _strided(ds, pad, shift))
    torch.cuda.synchronize()
    zero = torch.zeros((T, d), dtype=torch.float64)
    want, wdw, wdb, n, g, mg, mn = _norm_grad(x.double(), dy.double(), w.double(), mean, rstd,
                                              zero if ds is None else ds.double(), centre)
    # n: two roundings; g: one; the means: d + 3 of the terms' sizes; the rest a few
    eg, en = U32 * g.abs(), 2.1 * U32 * n.abs()
    emg = (d + 3) * U32 * g.abs().mean(1, keepdim=True) if centre else 0.0
    emn = (d + 6) * U32 * (g * n).abs().mean(1, keepdim=True)
    size = g.abs() + abs(mg) + (n * mn).abs()
    e = rstd * (eg + emg + en * mn.abs() + n.abs() * emn + 4 * U32 * size) + 2 * U32 * want.abs()
    _within(dx, want, e + _u(dtype) * (want.abs() + e) + _tiny(dtype), "dx")
    _within(dw, wdw, (T + 4) * U32 * (dy.double() * n).abs().sum(0) + 2.0 ** -149, "dweight")
    _within(db, wdb, (T + 1) * U32 * dy.double().abs().sum(0), "dbias")
    # each alone, and none of a weight
    only = pk.layernorm_backward(*args, need_dx=False, need_dbias=False)
    assert only[0] is None and only[2] is None
    _within(only[1], wdw, (T + 4) * U32 * (dy.double() * n).abs().sum(0) + 2.0 ** -149, "dweight alone")
    only = pk.layernorm_backward(*args, need_dweight=False, need_dbias=False)
    assert only[1] is None and only[2] is None
    plain = pk.layernorm_backward(gs, xs, torch.ones(d, device=DEV), f.mean, f.rstd)[0]
    assert torch.equal(pk.layernorm_backward(gs, xs, None, f.mean, f.rstd)[0], plain)


@pytest.mark.parametrize("centre", [True, False])
def test_layernorm_backward_against_differences(centre):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("layernorm differences", centre)
    T, d = 6, 40
    x, w, b, dy = _rand((T, d), 1), 1 + 0.1 * _rand((d,), 2), _rand((d,), 3), _rand((T, d), 4)
    x32, w32 = x.float(), w.float()

    def loss(x, w, b):
        m = x.mean(1, keepdim=True) if centre else 0.0
        y = (x - m) / torch.sqrt((x - m).square().mean(1, keepdim=True) + 1e-5) * w + b
        return float((y * dy.float().double()).sum())
    f = pk.layernorm(x32.to(DEV), w32.to(DEV), centre=centre)
    grads = pk.layernorm_backward(dy.float().to(DEV), x32.to(DEV), w32.to(DEV), f.mean, f.rstd)
    base = [x32.double(), w32.double(), b]
    for k, grad in enumerate(grads):
        v = _rand(base[k].shape, 10 + k)
        lo, hi = ([t + (e * v if i == k else 0) for i, t in enumerate(base)] for e in (-1e-5, 1e-5))
        diff = (loss(*hi) - loss(*lo)) / 2e-5
        got = float((grad.cpu().double() * v).sum())
        # fp32 gradients of sums of 6 x 40 terms around 1: 300 roundings of their sizes; differences: 1e-10 of third
        # derivatives
        assert abs(diff - got) <= 300 * U32 * float((grad.cpu().double() * v).abs().sum()) + 1e-7, k


# ---------------------------------------------------------------- vocabulary loss
def _head_inputs(T, d, V, dtype, seed=0):
    torch = _t()
    dt = _dtype(dtype)
    w = (_rand((V, d), seed + 1) * (2.5 / math.sqrt(d))).to(dt)
    tok = _tokens(T, V, seed + 2)
    x = (_rand((T, d), seed + 3) + torch.linspace(0, 2, T, dtype=torch.float64)[:, None] * w[tok.clamp(0, V - 1)].double()).to(dt)
    return x, w, tok


def _head_ref(x, w, tok):
    torch = _t()
    V = w.shape[0]
    z = x.double() @ w.double().t()
    size = x.double().abs() @ w.double().abs().t()
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = logp.exp()
    H = torch.special.entr(p).sum(1)
    asked = (tok >= 0) & (tok < V)
    at = logp.gather(1, tok.clamp(0, V - 1)[:, None])[:, 0]
    return z, size, lse, logp, p, H, asked, torch.where(asked, at, 0.0)


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V,pad,shift", HEAD)
def test_head_logprobs(dtype, T, d, V, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head", dtype, T, d, V, pad, shift)
    x, w, tok = _head_inputs(T, d, V, dtype)
    got = pk.head_logprobs(_strided(x, pad, shift), _strided(w, pad, shift), tok.to(DEV))
    torch.cuda.synchronize()
    z, size, lse, logp, p, H, asked, at = _head_ref(x, w, tok)
    ez = (d + 1) * U32 * size.amax(1)                        # of a logit
    # s = sum exp(z - m): V terms, each off by 2 ez, by the exponent's rounding |z - m| U32 (weighted with p: at most that of
    # the entropy and of log s) and by 4 U32; the parts' joins, a few roundings each level
    es = 2 * ez + (V + 40) * U32 + 4 * U32 * (1 + H)
    _within(got.lse, lse, ez + es + 2 * U32 * (lse.abs() + 1), "lse")
    _within(got.logprob, at, torch.where(asked, 2 * ez + es + 4 * U32 * (at.abs() + lse.abs() + 1), 0.0), "logprob")
    span = (z.amax(1) - z.amin(1)) + 1
    _within(got.entropy, H, 4 * es * span + 8 * U32 * (span + 1), "entropy")
    again = pk.head_logprobs(_strided(x, pad, shift), _strided(w, pad, shift), tok.to(DEV))
    assert all(torch.equal(a, b) for a, b in zip(got[:3], again[:3]))
    none = pk.head_logprobs(x.to(DEV), w.to(DEV))
    assert none.logprob is None
    _within(none.lse, lse, ez + es + 2 * U32 * (lse.abs() + 1), "lse without targets")


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("T,d,V,pad,shift", HEAD)
def test_head_logprobs_backward(dtype, entropy, T, d, V, pad, shift):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head backward", dtype, entropy, T, d, V, pad, shift)
    x, w, tok = _head_inputs(T, d, V, dtype)
    z, size, lse, logp, p, H, asked, _ = _head_ref(x, w, tok)
    gl = (-torch.rand((T,), generator=torch.Generator().manual_seed(9), dtype=torch.float64) / T).float()
    gh = (0.1 * _rand((T,), 10) / T).float() if entropy else None
    xs, ws = _strided(x, pad, shift), _strided(w, pad, shift)
    lse32, H32 = lse.float(), H.float()
    args = (xs, ws, tok.to(DEV), lse32.to(DEV), H32.to(DEV) if entropy else None, gl.to(DEV),
            gh.to(DEV) if entropy else None)
    dx, dw = pk.head_logprobs_backward(*args)
    torch.cuda.synchronize()
    g = torch.where(asked, gl.double(), 0.0)[:, None]
    one = (torch.arange(V)[None, :] == tok[:, None]).double()
    dz = g * (one - p)
    slope = g.abs() * (one + p)
    if entropy:
        e = gh.double()[:, None]
        dz = dz - e * p * (logp + H[:, None])
        slope = slope + e.abs() * p * (logp.abs() + H[:, None] + 1)
    # dz: p off by the logit's error, lse's rounding and exp's; then its own rounding to dtype (with the rests, T <= 64,
    # twice as many bits), below the range of f16 an absolute one of 2^-38 of the largest gradient
    ez = (d + 1) * U32 * size.amax(1, keepdim=True) + 2 * U32 * (lse.abs()[:, None] + logp.abs() + 2)
    u = _u(dtype)
    low = float((gl.abs().max() + (4 * gh.abs().max() if entropy else 0))) * 2.0 ** -37 if dtype == "f16" else 0.0
    edz = slope * (2 * ez + 8 * U32) + (u * u if T <= 64 else u) * dz.abs() + low
    sx, sw = (dz.abs() @ w.double().abs(), dz.abs().t() @ x.double().abs())
    for got, want, err, s, n in ((dx, dz @ w.double(), edz @ w.double().abs(), sx, V),
                                 (dw, dz.t() @ x.double(), edz.t() @ x.double().abs(), sw, T)):
        tol = err + (2 * n + 8) * U32 * (s + err)
        _within(got, want, tol + u * (want.abs() + tol) + _tiny(dtype), "dx" if n == V else "dw")
        # Roundings average: of numbers of any mantissa the error is 0.43 u of their root mean square (a step's
        # half is u at the lower end of a power of two, the mean square 1/12 step^2 over x^2 in [1, 4)), and so is that of n
        # independent ones within a share of 2 / sqrt(n) (their squares deviate by about their mean; four times that, halved by
        # the root).  The result's own are as many as it has entries.  dz's act on a whole row of dx, of which one in
        # four counts (one entry of dz is most of a row where the softmax is peaked); with the rests there are none.
        own = 0.44 * u * (1 + 2 / math.sqrt(want.numel()))
        of_dz = 0.44 * u * (1 + 2 / math.sqrt(T / 4)) if T > 64 else 0.0
        far, most = float((got.cpu().double() - want).norm()), math.hypot(own, of_dz) * float(want.norm())
        assert far <= most + _tiny(dtype) * math.sqrt(want.numel()) + float(tol.norm() if T <= 64 else 0.0), (far, most)
    only = pk.head_logprobs_backward(*args, need_dw=False)
    assert only[1] is None and torch.equal(only[0], dx)
    only = pk.head_logprobs_backward(*args, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dw)


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V,pad,shift", HEAD_LARGE)
def test_head_large(dtype, T, d, V, pad, shift):
    """Forward and backward against 64 bits on the GPU (its products in 64 bits are torch's)."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head large", dtype, T, d, V, pad, shift)
    x, w, tok = _head_inputs(T, d, V, dtype)
    xs, ws, tk = _strided(x, pad, shift), _strided(w, pad, shift), tok.to(DEV)
    xd, wd = x.to(DEV).double(), w.to(DEV).double()
    z = xd @ wd.t()
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    H = torch.special.entr(logp.exp()).sum(1)
    asked = (tk >= 0) & (tk < V)
    at = torch.where(asked, logp.gather(1, tk.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    got = pk.head_logprobs(xs, ws, tk)
    ez = float((d + 1) * U32 * (xd.abs().amax() * wd.abs().sum(1).amax()))   # (bounds of test_head_logprobs, the largest row's)
    es = 2 * ez + (V + 40) * U32 + 4 * U32 * (1 + H)
    span = (z.amax(1) - z.amin(1)) + 1
    for g, want, tol in ((got.lse, lse, ez + es + 2 * U32 * (lse.abs() + 1)), (got.entropy, H, 4 * es * span + 8 * U32 * (span + 1)),
                         (got.logprob, at, torch.where(asked, 2 * ez + es + 4 * U32 * (at.abs() + lse.abs() + 1), 0.0))):
        _within(g, want.cpu(), tol.cpu(), "forward")
    del z
    gl = (-torch.rand((T,), generator=torch.Generator().manual_seed(9)) / T).to(DEV)
    dx, dw = pk.head_logprobs_backward(xs, ws, tk, lse.float(), g_logprob=gl)
    again = pk.head_logprobs_backward(xs, ws, tk, lse.float(), g_logprob=gl)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    dz = logp.exp_().mul_(-torch.where(asked, gl.double(), 0.0)[:, None])
    # p's own error, of a logit's, of lse's rounding and of exp's, counts in full where 1 - p is small
    edz = dz.abs() * (2 * ez + 2 * U32 * (lse.abs()[:, None] + 30) + 8 * U32)
    dz[asked, tk[asked]] += gl.double()[asked]
    u = _u(dtype)
    for got, want in ((dx, dz @ wd), (dw, dz.t().contiguous() @ xd)):
        far = float((got.double() - want).norm())
        own = 0.44 * u * (1 + 2 / math.sqrt(want.numel()))             # (as in test_head_logprobs_backward)
        of_dz = 0.44 * u * (1 + 2 / math.sqrt(T / 4))
        assert far <= (math.hypot(own, of_dz) + 1e-6) * float(want.norm()) + _tiny(dtype) * math.sqrt(want.numel()), far
        # and no row is wrong: entrywise, a rounding of each term and of the result
        size = dz.abs() @ wd.abs() if got is dx else dz.abs().t().contiguous() @ xd.abs()
        of_p = edz @ wd.abs() if got is dx else edz.t().contiguous() @ xd.abs()
        low = float(gl.abs().max()) * 2.0 ** -37 * max(T, V) * float(xd.abs().max()) if dtype == "f16" else 0.0
        tol = 1.01 * (u * size + of_p + 2 * max(T, V) * U32 * size) + u * want.abs() + _tiny(dtype) + low
        bad = (got.double() - want).abs() > tol
        assert not bool(bad.any()), (got is dx, int(bad.sum()), float(((got.double() - want).abs() / tol).max()))
