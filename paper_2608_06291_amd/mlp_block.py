"""A gated MLP block quantised end to end: calibrated, rounded, served and judged.

The block of a pre-norm network is
  y = RMSNorm(x),  h = act(W_gate y) (.) W_up y,  out = x + W_down h.
Rounding its three matrices with BaKron and running the result takes every operator around
the solver:

  * calibration: `gated_mlp` gives h and the features of the MLP-local Hessians of W_up
    and W_gate (App. A); the loss's gradient at the logits (`token_logprobs_backward`)
    gives b, the gradient at the block's output, for the global Hessian of W_down;
    `gated_mlp_backward` takes b on to the layers before;
  * rounding: `mse_scales`, `factor`, `solve` for each matrix, `pack_codes`;
  * serving: `rmsnorm_quant` makes 8-bit rows, `linear` multiplies them with the codes, the
    activation, the gate's product and the residual in its epilogue;
  * judging: `token_logprobs` before and after.

  python -m paper_2608_06291_amd.mlp_block [--d 512] [--f 1376] [--vocab 4096] [--tokens 2048]
"""
from __future__ import annotations

from dataclasses import dataclass, field

from . import _lib


@dataclass
class GatedMLP:
    """The block in 16-bit floats.  norm: d fp32; w_gate, w_up: f x d; w_down: d x f."""
    norm: object
    w_gate: object
    w_up: object
    w_down: object
    act: str = "silu"
    eps: float = 1e-5

    def forward(self, x, features: bool = False):
        """(out, y, MlpFeatures or h) for x: T x d."""
        y = _lib.rmsnorm_quant(x, self.norm, eps=self.eps, quantise=False, with_y=True).y
        h = _lib.gated_mlp(y, self.w_gate, self.w_up, act=self.act, features=features)
        out = x + (h.h if features else h) @ self.w_down.t()
        return out, y, h

    def backward(self, x, y, b):
        """(dx, dw_gate, dw_up) from b, the gradient with respect to the block's output.  The
        norm's gradient, a small part of the work, is torch's."""
        dy, dw_gate, dw_up = _lib.gated_mlp_backward(b @ self.w_down, y, self.w_gate, self.w_up, act=self.act)
        xf, g = x.float(), dy.float() * self.norm
        r = (xf.square().mean(1, keepdim=True) + self.eps).rsqrt()
        dx = r * (g - xf * (r * r) * (g * xf).mean(1, keepdim=True))
        return (b.float() + dx).to(x.dtype), dw_gate, dw_up


@dataclass
class _Layer:
    codes: object      # PackedCodes
    scale: object      # m, or m x groups


@dataclass
class QuantisedMLP:
    """The same block on codes: three products of 8-bit rows."""
    norm: object
    gate: _Layer
    up: _Layer
    down: _Layer
    act: str
    eps: float
    group_size: int = 0
    values: dict = field(default_factory=dict)   # V of each matrix, for checks

    def forward(self, x, residual=None):
        """The block's output for the stream x (+ residual, added on the way in)."""
        r = _lib.rmsnorm_quant(x, self.norm, residual=residual, eps=self.eps)
        stream = x if residual is None else r.sum
        g, dt = self.group_size, x.dtype
        u = _lib.linear(r.q, r.scale, self.up.codes, self.up.scale, group_size=g, dtype=dt)
        h = _lib.linear(r.q, r.scale, self.gate.codes, self.gate.scale, group_size=g, act=self.act, other=u,
                        combine="mul", out=u)
        q = _lib.rmsnorm_quant(h, normalise=False)
        return _lib.linear(q.q, q.scale, self.down.codes, self.down.scale, group_size=g, other=stream, dtype=dt)


def quantise(block: GatedMLP, x, b, bits: int = 4, damp: float = 0.01, group_size: int = 0) -> QuantisedMLP:
    """Rounds the block's matrices from calibration tokens x (N x d) and the gradients b
    (N x d) of the loss at its output."""
    _, y, feat = block.forward(x, features=True)
    yf, hf, down = y.float(), feat.h.float(), block.w_down.float().contiguous()
    values = {}

    def round_to_codes(name, w, A, B):
        w = w.float().contiguous()
        scale = _lib.mse_scales(w, bits, group_size=group_size, grid=100, maxshrink=0.5)
        f = _lib.factor(A, B, damp)
        codes, values[name] = _lib.solve(w, f, bits, scale, group_size=group_size)
        f.close()
        return _Layer(_lib.pack_codes(codes, 4 if bits <= 4 else 8), scale)

    up = round_to_codes("up", block.w_up, *_lib.mlp_local_factors(yf, feat.up, down))
    gate = round_to_codes("gate", block.w_gate, *_lib.mlp_local_factors(yf, feat.gate, down))
    dn = round_to_codes("down", block.w_down, *_lib.kron_factors(hf, b.float().contiguous()))
    return QuantisedMLP(block.norm, gate, up, dn, block.act, block.eps, group_size, values)


def run(d: int = 512, f: int = 1376, vocab: int = 4096, tokens: int = 2048, bits: int = 4, group_size: int = 0,
        seed: int = 0, device: str = "cuda:0"):
    """Calibrates, rounds and judges one random block before a random vocabulary matrix;
    returns what main() prints."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=device) * scale).to(torch.bfloat16)

    block = GatedMLP(1 + 0.1 * torch.randn((d,), generator=gen, device=device), rand(f, d, scale=d ** -0.5),
                     rand(f, d, scale=d ** -0.5), rand(d, f, scale=f ** -0.5))
    head = rand(vocab, d, scale=2.0 * d ** -0.5)
    x = rand(tokens, d)
    out, y, _ = block.forward(x)
    logits = out @ head.t()
    # tokens as the float block would draw them
    noise = torch.rand((tokens, vocab), generator=gen, device=device).clamp_(1e-9, 1 - 1e-7)
    target = (logits.float() - torch.log(-torch.log(noise))).argmax(1)
    before = _lib.token_logprobs(logits, target, top=1)
    dz = _lib.token_logprobs_backward(logits, target, before.lse, g_logprob=torch.full((tokens,), -1.0, device=device))
    b = dz @ head
    dx, dw_gate, dw_up = block.backward(x, y, b)
    served = quantise(block, x, b, bits=bits, group_size=group_size)
    after = _lib.token_logprobs(served.forward(x) @ head.t(), target, top=1)
    return dict(block=block, served=served, head=head, x=x, target=target, before=before, after=after, b=b, dx=dx,
                dw_gate=dw_gate, dw_up=dw_up,
                nll_before=float(-before.logprob.mean()), nll_after=float(-after.logprob.mean()),
                same_top=float((before.top_index == after.top_index).float().mean()))


def main():
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("d", 512), ("f", 1376), ("vocab", 4096), ("tokens", 2048), ("bits", 4), ("group-size", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    r = run(a.d, a.f, a.vocab, a.tokens, a.bits, a.group_size)
    print(f"negative log likelihood a token: {r['nll_before']:.4f} in 16-bit floats, {r['nll_after']:.4f} with "
          f"{a.bits}-bit codes and 8-bit rows; same most likely token: {100 * r['same_top']:.1f}%")


if __name__ == "__main__":
    main()
