"""GPU tests of the operators around a quantised layer where numbers leave the middle of
their range: the smallest and largest ones, a common offset, the tails of the activations.

Tolerances as in test_gpu_operators.py: bounds on the roundings that the header allows.
"""
import pytest

from test_gpu_operators import U32, _say, _t

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
