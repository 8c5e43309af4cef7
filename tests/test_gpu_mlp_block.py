"""GPU test of the quantised gated MLP block: every operator around the solver in one
path, against a 64-bit evaluation of the same block from the rounded values V, and the
log probabilities before and after."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,group_size", [(4, 0), (4, 64), (8, 0)])
def test_quantised_block(bits, group_size):
    import torch
    from paper_2608_06291_amd import mlp_block
    print("block", bits, group_size, flush=True)
    r = mlp_block.run(d=200, f=330, vocab=600, tokens=512, bits=bits, group_size=group_size, seed=3)
    s, blk, x = r["served"], r["block"], r["x"]
    got = s.forward(x)
    torch.cuda.synchronize()
    # the same block in 64 bits on V, with rows rounded to 8 bits as the norm rounds them
    V = {k: v.cpu().double() for k, v in s.values.items()}
    xd = x.cpu().double()

    def rows8(y):
        sc = y.abs().amax(1, keepdim=True) / 127
        return torch.round(y / sc) * sc
    y = xd / torch.sqrt(xd.square().mean(1, keepdim=True) + s.eps) * s.norm.cpu().double()
    q = rows8(y)
    g, u = q @ V["gate"].t(), (q @ V["up"].t()).to(torch.bfloat16).double()
    h = (g * torch.sigmoid(g) * u).to(torch.bfloat16).double()
    want = xd + rows8(h) @ V["down"].t()
    # One 8-bit code off by one step (a tie decided by an fp32 rounding) or one bf16 rounding of h
    # the other way moves an output by at most a step times a weight; output itself is rounded to bf16.
    step = (h.abs().amax(1, keepdim=True) / 127) * V["down"].abs().amax() * 2
    err = (got.cpu().double() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + step + 1e-3).all()), float(err.max())
    rel = float(err.norm() / want.norm())
    assert rel < 3e-3, rel
    # a residual added on the way in is the same as one added before
    half = (x.float() * 0.5).to(x.dtype)
    assert torch.equal(s.forward(half, residual=half), s.forward(half + half))
    # rounding costs little likelihood, less with more bits
    assert math.isfinite(r["nll_after"])
    assert r["nll_after"] - r["nll_before"] < (0.02 if bits == 8 else 0.5), (r["nll_before"], r["nll_after"])
    assert r["same_top"] > (0.9 if bits == 8 else 0.4)


def test_block_gradients_against_differences():
    """The gradient that the block hands on, against differences of the 64-bit loss."""
    import torch
    from paper_2608_06291_amd import mlp_block
    print("block gradients", flush=True)
    r = mlp_block.run(d=72, f=104, vocab=90, tokens=40, bits=8, seed=5)
    blk, head, x, target = r["block"], r["head"].cpu().double(), r["x"].cpu().double(), r["target"].cpu()
    norm, wg, wu, wd = (t.cpu().double() for t in (blk.norm, blk.w_gate, blk.w_up, blk.w_down))

    def loss(x, wg, wu):
        y = x / torch.sqrt(x.square().mean(1, keepdim=True) + blk.eps) * norm
        g = y @ wg.t()
        out = x + (g * torch.sigmoid(g) * (y @ wu.t())) @ wd.t()
        return float(torch.nn.functional.cross_entropy(out @ head.t(), target, reduction="sum"))
    base = [x, wg, wu]
    for k, grad in enumerate((r["dx"], r["dw_gate"], r["dw_up"])):
        gen = torch.Generator().manual_seed(k)
        v = torch.randn(base[k].shape, generator=gen, dtype=torch.float64)
        lo, hi = ([t + (e * v if i == k else 0) for i, t in enumerate(base)] for e in (-1e-5, 1e-5))
        diff = (loss(*hi) - loss(*lo)) / 2e-5
        g = grad.cpu().double()
        # every product on the way (logits, dz, b, dh, dG, dU, the result) is rounded to bf16,
        # u = 2^-8 each, seven of them, independent from entry to entry: the sum over n entries is
        # off by about u sqrt(7) of the root of the sum of squares; five times that
        size = float((g * v).norm())
        assert abs(diff - float((g * v).sum())) <= 5 * 2.0 ** -8 * math.sqrt(7) * size, k
