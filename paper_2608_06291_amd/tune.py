"""Tuning what rounding leaves in floats: the vocabulary matrix and the norms.

A network of one gated MLP block between a table and the same table as vocabulary matrix:
  x = s E[tokens],   out = block(x),   logits = RMSNorm(out) E^T
Once the block's matrices are rounded, its norm, the last norm and E are still floats, and a few steps
against the loss move them to where the rounded matrices want them.  A step takes every operator at
the ends of a network:

  * `embedding` -> the block -> `layernorm` -> `head_logprobs`: the loss, without logits;
  * `head_logprobs_backward` -> `layernorm_backward` -> the block's gradients (its matrices as they
    were rounded) -> `embedding_backward`, on top of the same matrix's gradient at the other end.

  python -m paper_2608_06291_amd.tune [--d 512] [--f 1376] [--vocab 4096] [--tokens 2048] [--steps 8]
"""
from __future__ import annotations

from dataclasses import dataclass

from . import _lib, mlp_block


@dataclass
class TiedNetwork:
    """table: V x d in 16-bit floats; final: d fp32; block: a GatedMLP."""
    table: object
    block: mlp_block.GatedMLP
    final: object
    eps: float = 1e-5

    @property
    def scale(self):
        return float(self.table.shape[1]) ** 0.5

    def forward(self, tokens):
        """(x, out, y, last): the block's input, output and normed input, and the last norm."""
        x = _lib.embedding(tokens, self.table, scale=self.scale)
        out, y, _ = self.block.forward(x)
        return x, out, y, _lib.layernorm(out, self.final, eps=self.eps, centre=False)

    def logprobs(self, tokens, target):
        """TokenLogprobs of the targets (T int64, outside the vocabulary: ignored)."""
        return _lib.head_logprobs(self.forward(tokens)[3].y, self.table, target)

    def gradients(self, tokens, target, g_logprob=None):
        """(TokenLogprobs, gradients) of sum_t g_logprob_t logprob_t, with g_logprob None of minus the mean over
        the targets that count: a dict with `table` in its type, `norm` and `final` in fp32."""
        import torch
        x, out, y, last = self.forward(tokens)
        lp = _lib.head_logprobs(last.y, self.table, target)
        if g_logprob is None:
            count = ((target >= 0) & (target < self.table.shape[0])).sum().clamp(min=1)
            g_logprob = (-1.0 / count).expand(tokens.shape[0]).to(torch.float32).contiguous()
        dlast, dtable = _lib.head_logprobs_backward(last.y, self.table, target, lp.lse, g_logprob=g_logprob)
        dout, dfinal, _ = _lib.layernorm_backward(dlast, out, self.final, None, last.rstd, need_dbias=False)
        dx, _, _, dnorm = self.block.gradients(x, y, dout, need_dw=False)
        dtable = _lib.embedding_backward(dx, tokens, self.table.shape[0], scale=self.scale, base=dtable, out=dtable)
        return lp, {"table": dtable, "norm": dnorm, "final": dfinal}

    def step(self, tokens, target, rate: float):
        """One step of gradient descent on the three; returns the mean negative log probability before it."""
        lp, g = self.gradients(tokens, target)
        asked = (target >= 0) & (target < self.table.shape[0])
        loss = -lp.logprob.sum() / asked.sum().clamp(min=1)
        self.table = (self.table.float() - rate * g["table"].float()).to(self.table.dtype)
        self.block.norm = self.block.norm - rate * g["norm"]
        self.final = self.final - rate * g["final"]
        return loss


def run(d: int = 512, f: int = 1376, vocab: int = 4096, tokens: int = 2048, bits: int = 3, steps: int = 8,
        rate: float = 0.5, seed: int = 0, device: str = "cuda:0"):
    """Rounds a random network's block to `bits` and tunes its floats against tokens that the network drew before
    it was rounded; returns what main() prints."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=device) * scale).to(torch.bfloat16)

    # (w_down so large that the block's output, not the token that came in, is most of the stream)
    block = mlp_block.GatedMLP(1 + 0.1 * torch.randn((d,), generator=gen, device=device), rand(f, d, scale=d ** -0.5),
                               rand(f, d, scale=d ** -0.5), rand(d, f, scale=16.0 * f ** -0.5))
    net = TiedNetwork(rand(vocab, d, scale=2.0 * d ** -0.5), block, torch.ones(d, device=device))
    text = torch.randint(0, vocab, (tokens,), generator=gen, device=device)
    x, out, _, last = net.forward(text)
    noise = torch.rand((tokens, vocab), generator=gen, device=device).clamp_(1e-9, 1 - 1e-7)
    target = ((last.y @ net.table.t()).float() - torch.log(-torch.log(noise))).argmax(1)
    del noise
    lp = net.logprobs(text, target)
    g = torch.full((tokens,), -1.0 / tokens, device=device)
    dlast, _ = _lib.head_logprobs_backward(last.y, net.table, target, lp.lse, g_logprob=g, need_dw=False)
    b = _lib.layernorm_backward(dlast, out, net.final, None, last.rstd, need_dweight=False, need_dbias=False)[0]
    served = mlp_block.quantise(block, x, b, bits=bits)
    rounded = mlp_block.GatedMLP(block.norm, *(served.values[k].to(torch.bfloat16) for k in ("gate", "up", "down")),
                                 act=block.act, eps=block.eps)
    net.block = rounded
    losses = [float(net.step(text, target, rate)) for _ in range(steps)]
    return dict(net=net, text=text, target=target, nll_float=float(-lp.logprob.mean()), losses=losses,
                nll_tuned=float(-net.logprobs(text, target).logprob.mean()))


def main():
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("d", 512), ("f", 1376), ("vocab", 4096), ("tokens", 2048), ("bits", 3), ("steps", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=0.5)
    a = ap.parse_args()
    r = run(a.d, a.f, a.vocab, a.tokens, a.bits, a.steps, a.rate)
    print(f"negative log likelihood a token: {r['nll_float']:.4f} in 16-bit floats, {r['losses'][0]:.4f} with the block "
          f"in {a.bits} bits, {r['nll_tuned']:.4f} after {a.steps} steps on the norms and the "
          "vocabulary matrix (of the tokens that these were tuned on)")


if __name__ == "__main__":
    main()
