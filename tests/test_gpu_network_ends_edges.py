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
