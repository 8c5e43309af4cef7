"""GPU tests of a network's floats tuned around a rounded block: every operator at the ends of a network in one
path, its gradients against differences of the same loss in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _network(V, d, f, seed):
    import torch
    from paper_2608_06291_amd import mlp_block, tune
    gen = torch.Generator().manual_seed(seed)

    def rand(*shape, scale):
        return (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16).to("cuda:0")
    block = mlp_block.GatedMLP((1 + 0.1 * torch.randn(d, generator=gen)).to("cuda:0"), rand(f, d, scale=d ** -0.5),
                               rand(f, d, scale=d ** -0.5), rand(d, f, scale=f ** -0.5))
    return tune.TiedNetwork(rand(V, d, scale=d ** -0.5), block, (1 + 0.1 * torch.randn(d, generator=gen)).to("cuda:0"))


def _loss(net, tokens, target, g, table, norm, final):
    """sum g logprob in 64 bits on the CPU."""
    import torch
    blk = net.block
    wg, wu, wd = (t.cpu().double() for t in (blk.w_gate, blk.w_up, blk.w_down))
    V, d = table.shape
    asked = (tokens >= 0) & (tokens < V)
    x = torch.where(asked[:, None], table[tokens.clamp(0, V - 1)] * d ** 0.5, 0.0)

    def rms(x):
        return x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5)
    y = rms(x) * norm
    h = y @ wg.t()
    out = x + (h * torch.sigmoid(h) * (y @ wu.t())) @ wd.t()
    logp = torch.log_softmax((rms(out) * final) @ table.t(), 1)
    ok = (target >= 0) & (target < V)
    return float((torch.where(ok, logp.gather(1, target.clamp(0, V - 1)[:, None])[:, 0], 0.0) * g).sum())


@pytest.mark.parametrize("V,d,f,T", [(90, 72, 104, 40), (301, 130, 70, 77)])
def test_gradients_against_differences(V, d, f, T):
    import torch
    print("tune", V, d, f, T, flush=True)
    net = _network(V, d, f, 4)
    gen = torch.Generator().manual_seed(5)
    tokens, target = (torch.randint(0, V, (T,), generator=gen) for _ in range(2))
    tokens[::9] = 7          # one token many times
    tokens[3], target[5], target[6] = -1, -100, V
    g = torch.rand((T,), generator=gen)
    lp, grads = net.gradients(tokens.cuda(), target.cuda(), g.cuda())
    torch.cuda.synchronize()
    base = {"table": net.table.cpu().double(), "norm": net.block.norm.cpu().double(), "final": net.final.cpu().double()}
    for k, name in enumerate(base):
        v = torch.randn(base[name].shape, generator=torch.Generator().manual_seed(k), dtype=torch.float64)
        lo, hi = (_loss(net, tokens, target, g.double(), **{n: t + (e * v if n == name else 0) for n, t in base.items()})
                  for e in (-1e-5, 1e-5))
        diff, got = (hi - lo) / 2e-5, grads[name].cpu().double()
        # every tensor on the way (x, y, h, out, the last norm, dz, dlast, dout, b W_down, dG, dU, dx, the result) is rounded to
        # bf16, u = 2^-8 each, 13 of them, independent from entry to entry: the sum over the entries is off by about
        # u sqrt(13) of the root of the sum of squares; five times that
        size = float((got * v).norm())
        assert abs(diff - float((got * v).sum())) <= 5 * 2.0 ** -8 * math.sqrt(13) * size, name
    # the loss itself: each row's logits are off by the rounding of a few rows of d entries
    want = _loss(net, tokens, target, g.double(), **base)
    assert abs(float((lp.logprob.cpu().double() * g.double()).sum()) - want) <= 2.0 ** -8 * 6 * T


def test_step_and_command():
    import torch
    from paper_2608_06291_amd import tune
    print("tune run", flush=True)
    r = tune.run(d=128, f=200, vocab=700, tokens=300, bits=4, steps=2, seed=1)
    assert len(r["losses"]) == 2 and all(math.isfinite(v) for v in r["losses"] + [r["nll_float"], r["nll_tuned"]])
    net = r["net"]
    before = [t.clone() for t in (net.table, net.block.norm, net.final)]
    lp, g = net.gradients(r["text"], r["target"])
    net.step(r["text"], r["target"], 0.25)
    assert torch.equal(net.table, (before[0].float() - 0.25 * g["table"].float()).to(before[0].dtype))
    assert torch.equal(net.block.norm, before[1] - 0.25 * g["norm"]) and torch.equal(net.final, before[2] - 0.25 * g["final"])


def test_block_gradients_of_any_layout():
    """Transposed, broadcast and graph-bearing rows give what contiguous ones do."""
    import torch
    net = _network(90, 72, 104, 3)
    gen = torch.Generator().manual_seed(4)
    x, b = ((torch.randn((40, 72), generator=gen) * 0.5).to(torch.bfloat16).to("cuda:0") for _ in range(2))
    y = net.block.forward(x)[1]
    want = net.block.gradients(x, y, b)
    flat = b[:1].expand(40, 72)
    want_flat = net.block.gradients(x, y, flat.contiguous())
    turned = lambda t: t.t().contiguous().t()
    for got, ref in ((net.block.gradients(turned(x), y, turned(b)), want), (net.block.gradients(x, y, flat), want_flat),
                     (net.block.gradients(x.clone().requires_grad_(), y, b), want)):
        for g, r in zip(got, ref):
            assert torch.equal(g, r) and not g.requires_grad
    assert all(torch.equal(g, r) for g, r in zip(net.block.backward(turned(x), y, turned(b)), want[:3]))
