"""GPU tests of what the binding of the operators around a quantised layer takes and refuses."""
import pytest

from test_gpu_operators import _padded_rows, _say, _t

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _layer(m=6, n=256, T=3):
    import paper_2608_06291_amd as pk
    torch = _t()
    g = torch.Generator().manual_seed(1)
    codes = torch.randint(-7, 8, (m, n), generator=g, dtype=torch.int8)
    return _padded_rows(torch.randint(-127, 128, (T, n), generator=g, dtype=torch.int8)), codes, pk.pack_codes(codes.to(DEV))


def test_linear_takes_scales_in_their_shape_only():
    """As many scales in another order would give other products."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear, scales' shape")
    q, codes, w = _layer()
    m = codes.shape[0]
    scale = torch.rand((m, 4), device=DEV) + 0.5
    want = (q.cpu().double().view(3, 1, 4, 64) * codes.double().view(1, m, 4, 64)).sum(3) * scale.cpu().double()
    y = pk.linear(q, None, w, scale, group_size=64, dtype=torch.float32)
    assert float((y.cpu().double() - want.sum(2)).abs().max()) <= 1e-6 * float(want.abs().sum(2).max())
    for bad in (scale.t().contiguous(), scale.flatten(), scale.view(2, 12), scale[:, :, None]):
        with pytest.raises(ValueError):
            pk.linear(q, None, w, bad, group_size=64)
    one = torch.rand(m, device=DEV)
    want = pk.linear(q, None, w, one)
    assert torch.equal(pk.linear(q, None, w, one[:, None]), want)                    # m x 1
    assert torch.equal(pk.linear(q, None, w, one[:, None], group_size=256), want)    # one group
    for bad in (one[None], one.view(2, 3)):
        with pytest.raises(ValueError):
            pk.linear(q, None, w, bad)
