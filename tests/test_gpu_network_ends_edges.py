"""GPU tests of the operators at the ends of a network where calls of one kind meet inputs of another: rows that ask for
nothing beside rows that do, results in the place of inputs, statistics that have to be better than a bound of the worst
case says."""
import math

import pytest

from network_ends_sizes import HEAD, HEAD_LARGE
from test_gpu_network_ends import DEV, U32, _dtype, _head_inputs, _rand, _say, _strided, _t, _tiny, _u

pytestmark = pytest.mark.gpu


# every place that the scale of half precision is taken in: up to 16 and 32 rows, few rows of few tokens, 65 to 512 rows
# in tiles, more; each with one and two results
@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V", [(5, 256, 900), (20, 256, 900), (6, 5, 900), (40, 256, 900), (40, 520, 300), (200, 256, 900), (600, 256, 900)])
def test_rows_that_ask_for_nothing_do_not_scale(dtype, T, d, V):
    """Whatever comes in at a row without a target, or without a finite logit, changes nothing of the others."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head, rows without a target", dtype, T, d, V)
    x, w, tok = (t.to(DEV) for t in _head_inputs(T, d, V, dtype))
    lp = pk.head_logprobs(x, w, tok)
    lse, H = lp.lse.clone(), lp.entropy.clone()
    tok[1], tok[T - 1], tok[2] = -100, V, V // 3
    lse[2], H[2] = -math.inf, 0.0        # logits of -inf throughout
    g = torch.Generator().manual_seed(3)
    gl, gh = (((torch.rand((T,), generator=g) - 0.5) / T).to(DEV) for _ in range(2))
    nothing = (tok < 0) | (tok >= V)
    for entropy in (False, True):
        want = None
        for size in (0.0, 1e30, -1e4, 3e38):
            a, b = gl.clone(), gh.clone()
            a[nothing] = size
            a[2] = b[2] = size
            args = (x, w, tok, lse, H if entropy else None, a, b if entropy else None)
            got = pk.head_logprobs_backward(*args)
            want = got if want is None else want
            assert bool(want[0][0].any()) and bool(want[1].any())
            for p, q in zip(got, want):
                assert torch.equal(p, q), (entropy, size)
            assert torch.equal(pk.head_logprobs_backward(*args, need_dw=False)[0], want[0])
            assert torch.equal(pk.head_logprobs_backward(*args, need_dx=False)[1], want[1])
    # without gradients of log probabilities the targets ask for nothing either way
    got = [pk.head_logprobs_backward(x, w, t, lse, H, None, gh) for t in (tok, None)]
    assert all(torch.equal(p, q) for p, q in zip(*got))


def _block(d, f, eps, dtype="bf16", seed=0):
    from paper_2608_06291_amd import mlp_block
    torch = _t()
    dt = _dtype(dtype)
    w = [(_rand(s, seed + k) * s[1] ** -0.5).to(dt).to(DEV) for k, s in enumerate(((f, d), (f, d), (d, f)))]
    return mlp_block.GatedMLP((1 + 0.1 * _rand((d,), seed + 5)).float().to(DEV), *w, eps=eps)


def _block_gradients(blk, x, b, dy):
    """(dx, bound of its error, dnorm, bound) of the block's norm from dy, in 64 bits."""
    torch = _t()
    xd, g, bd, norm = x.cpu().double(), dy.cpu().double(), b.cpu().double(), blk.norm.cpu().double()
    T, d = xd.shape
    ms = xd.square().mean(1, keepdim=True) + float(torch.tensor(blk.eps, dtype=torch.float32))
    r = torch.where(ms > 0, ms.rsqrt(), 0.0)
    n, gw = xd * r, g * norm
    mn = (gw * n).mean(1, keepdim=True)
    dx, dnorm = r * (gw - n * mn) + bd, (g * n).sum(0)
    # rstd: its sum's d roundings, halved by the root, and four more; n two more; g one; the mean d + 6 of its terms' sizes
    er = (d / 2 + 4) * U32
    en = (er + 2.1 * U32) * n.abs()
    size = gw.abs() + (n * mn).abs()
    e = r * (U32 * gw.abs() + en * mn.abs() + n.abs() * ((d + 6) * U32 + er + 3 * U32) * (gw * n).abs().mean(1, keepdim=True)
             + (4 * U32 + er) * size) + 2 * U32 * dx.abs()
    return dx, e, dnorm, ((T + 4) * U32 + er) * (g * n).abs().sum(0) + 2.0 ** -149


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-5])
@pytest.mark.parametrize("T,d,f", [(1, 64, 96), (40, 72, 104), (300, 130, 70)])
def test_block_gradients_of_any_eps(eps, dtype, T, d, f):
    """A block whose forward pass runs has its gradients, also with no eps and a row of zeros (which it leaves as they are)."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("block", dtype, eps, T, d, f)
    blk = _block(d, f, eps, dtype)
    x, b = (_rand((T, d), k).to(_dtype(dtype)).to(DEV) for k in (1, 2))
    if T > 2:
        x[2] = 0
    out, y, h = blk.forward(x)
    assert bool(torch.isfinite(out).all())
    dx, dw_gate, dw_up, dnorm = blk.gradients(x, y, b)
    dy = pk.gated_mlp_backward(b @ blk.w_down, y, blk.w_gate, blk.w_up, act=blk.act)
    assert torch.equal(dw_gate, dy[1]) and torch.equal(dw_up, dy[2])
    want, e, wnorm, en = _block_gradients(blk, x, b, dy[0])
    for got, w, lim in ((dx, want, e + _u(dtype) * (want.abs() + e) + _tiny(dtype)), (dnorm, wnorm, en)):
        assert bool(((got.cpu().double() - w).abs() <= lim).all()), float(((got.cpu().double() - w).abs() / lim).max())
    if T > 2 and eps == 0.0:
        assert torch.equal(dx[2], b[2])
    assert all(torch.equal(p, q) for p, q in zip(blk.backward(x, y, b), (dx, dw_gate, dw_up)))


@pytest.mark.parametrize("stream", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_block_gradients_of_a_stream_of_another_type(dtype, stream):
    """x of any type beside a block in 16 bits: dx in x's type, rounded once."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("block, stream", dtype, stream)
    T, d, f = 70, 130, 72
    blk = _block(d, f, 1e-5, dtype)
    x, b = _rand((T, d), 1).to(_dtype(stream)).to(DEV), _rand((T, d), 2).to(_dtype(dtype)).to(DEV)
    y = blk.forward(x.to(_dtype(dtype)))[1]
    dx, dw_gate, dw_up, dnorm = blk.gradients(x, y, b)
    assert dx.dtype == x.dtype and dw_gate.dtype == b.dtype and dnorm.dtype == torch.float32
    dy = pk.gated_mlp_backward(b @ blk.w_down, y, blk.w_gate, blk.w_up, act=blk.act)[0]
    want, e, wnorm, en = _block_gradients(blk, x, b, dy)
    e = e + U32 * (want.abs() + e) if stream != dtype else e   # (32 bits on the way)
    for got, w, lim in ((dx, want, e + _u(stream) * (want.abs() + e) + _tiny(stream)), (dnorm, wnorm, en)):
        assert bool(((got.cpu().double() - w).abs() <= lim).all()), float(((got.cpu().double() - w).abs() / lim).max())
    assert torch.equal(blk.backward(x, y, b)[0], dx)


@pytest.mark.parametrize("columns", [True, False])
@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("T,d", [(1, 64), (5, 131), (32, 1001), (33, 1001), (300, 1001), (3000, 72), (40, 20000), (300, 20001)])
def test_norm_gradients_in_place(dtype, T, d, columns):
    """dx in the place of dy, of x and of d_sum (through the C entry): the same results as beside them."""
    import ctypes

    import paper_2608_06291_amd as pk
    torch = _t()
    _say("layernorm backward in place", dtype, T, d, columns)
    lib, dt = pk.load(), _dtype(dtype)
    st = torch.cuda.current_stream().cuda_stream
    x, dy, ds = (_rand((T, d), k).to(dt).to(DEV) for k in (1, 2, 3))
    w = (1 + 0.1 * _rand((d,), 4)).float().to(DEV)
    f = pk.layernorm(x, w)
    want = pk.layernorm_backward(dy, x, w, f.mean, f.rstd, d_sum=ds, need_dweight=columns, need_dbias=columns)
    for place in range(3):
        rows = [t.clone() for t in (dy, x, ds)]
        sums = torch.full((2, d), 9.0, device=DEV)
        args = [rows[0].data_ptr(), d, rows[1].data_ptr(), d, {"f32": 0, "bf16": 2}[dtype], T, d, w.data_ptr(), f.mean.data_ptr(), f.rstd.data_ptr(),
                rows[2].data_ptr(), d, rows[place].data_ptr(), d, *(sums[k].data_ptr() if columns else None for k in range(2))]
        size = ctypes.c_size_t(0)
        assert lib.bakron_layernorm_backward(*args, None, ctypes.byref(size), st) == 0
        work = torch.empty(size.value + 256, dtype=torch.uint8, device=DEV)
        assert lib.bakron_layernorm_backward(*args, work.data_ptr(), ctypes.byref(size), st) == 0
        torch.cuda.synchronize()
        for k, t in enumerate((dy, x, ds)):
            assert torch.equal(rows[k], want[0] if k == place else t), (place, k)
        if columns:
            assert torch.equal(sums[0], want[1]) and torch.equal(sums[1], want[2]), place


def _walk(x, w, z):
    """Errors of fp32 logits as a random walk: each of d roundings is off by U32 of a partial sum at most, which lies between 0
    and z but for a few times the root of the sum of squares; independent ones add up to the root of their number.  Six times
    that, for the largest of many."""
    return 6 * x.shape[1] ** 0.5 * U32 * ((x.square() @ w.square().t()).sqrt() + z.abs())


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V,pad,shift", HEAD + HEAD_LARGE)
def test_head_statistics_as_good_as_their_sums(dtype, T, d, V, pad, shift):
    """lse, log probability and entropy within what roundings leave on the average, far below their own sizes: the bounds of the
    worst case would let whole nats of the entropy pass for long rows."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head statistics", dtype, T, d, V, pad, shift)
    x, w, tok = _head_inputs(T, d, V, dtype)
    xs, ws, tk = _strided(x, pad, shift), _strided(w, pad, shift), tok.to(DEV)
    got = pk.head_logprobs(xs, ws, tk)
    wd = w.to(DEV).double()
    for rows in torch.arange(T, device=DEV).split(1024):
        xd, t = x.to(DEV)[rows].double(), tk[rows]
        z = xd @ wd.t()
        ez = _walk(xd, wd, z)
        top = z.amax(1)
        lse = torch.logsumexp(z, 1)
        logp = z.sub_(lse[:, None])
        p = logp.exp()
        H = torch.special.entr(p).sum(1)
        # what the logits' errors make of lse and of the entropy, to the first order (the second is their square)
        of_lse, of_H = (p * ez).sum(1), (p * (logp + H[:, None]).abs() * ez).sum(1)
        asked = (t >= 0) & (t < V)
        k = t.clamp(0, V - 1)[:, None]
        at, ez_at = logp.gather(1, k)[:, 0], ez.gather(1, k)[:, 0]
        # the sums of V positive terms, a walk as well (four times the root of V), with 40 levels of joins and exp's 4 U32 and
        # those of its argument's rounding
        mean = (p * (top[:, None] - lse[:, None] - logp)).sum(1)           # sum p (m - z)
        es = (4 * V ** 0.5 + 40 + 4 * (1 + mean)) * U32
        second = (p * ez.square()).sum(1)
        for g, want, tol in ((got.lse, lse, of_lse + second + es + 2 * U32 * (lse.abs() + 1)),
                             (got.logprob, torch.where(asked, at, 0.0),
                              torch.where(asked, ez_at + of_lse + second + es + 4 * U32 * (at.abs() + 1), 0.0)),
                             (got.entropy, H, of_H + (2 + H) * second + es * (2 + mean) + 8 * U32 * (1 + mean + H))):
            far = (g[rows].double() - want).abs()
            assert bool((far <= tol).all()), float((far / tol.clamp(min=1e-300)).max())
        if V > 1000:
            # the bound says something of each row: 1% of its entropy, or of one nat where the entropy is less (it goes to 0 with
            # 1 - p of the row's token, the roundings of log s and of the mean, at 4 sqrt(V) U32 > 7e-6, do not)
            assert bool((tol < 0.01 * H.clamp(min=1.0)).all()), float(tol.max())
        del z, logp, p, ez


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V", [(2100, 520, 33000), (70, 1001, 67201), (2048, 1024, 16384), (600, 72, 9001)])
def test_head_large_gradients_of_entropies(dtype, T, d, V):
    """Gradients of log probabilities and entropies together, and of entropies alone, over tiles, pieces and parts."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head large, entropy", dtype, T, d, V)
    x, w, tok = (t.to(DEV) for t in _head_inputs(T, d, V, dtype))
    lp = pk.head_logprobs(x, w, tok)
    xd, wd = x.double(), w.double()
    logp = torch.log_softmax(xd @ wd.t(), 1)
    p = logp.exp()
    H = torch.special.entr(p).sum(1)
    g = torch.Generator().manual_seed(9)
    gl, gh = (((torch.rand((T,), generator=g) - 0.5) / T).to(DEV) for _ in range(2))
    asked = (tok >= 0) & (tok < V)
    for a in (gl, None):
        dz = -p * (gh.double()[:, None] * (logp + H[:, None]))
        if a is not None:
            ga = torch.where(asked, a.double(), 0.0)
            dz -= p * ga[:, None]
            dz[asked, tok[asked]] += ga[asked]
        u = _u(dtype)
        for got, want in zip(pk.head_logprobs_backward(x, w, tok, lp.lse, lp.entropy, a, gh), (dz @ wd, dz.t().contiguous() @ xd)):
            far = float((got.double() - want).norm())
            # one rounding of the result and one of dz, 0.43 u of a root mean square each, of as many numbers as there are
            # entries and rows (one in four of which counts); statistics in fp32 are 1e-3 of that
            own, of_dz = (0.44 * u * (1 + 2 / math.sqrt(n)) for n in (want.numel(), T / 4))
            assert far <= (math.hypot(own, of_dz) + 1e-5) * float(want.norm()) + _tiny(dtype) * math.sqrt(want.numel()), far / float(want.norm())
