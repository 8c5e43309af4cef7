"""GPU tests of the operators around a quantised layer at sizes whose counts and offsets pass 31 or 32 bits."""
import pytest

from test_gpu_operators import U32, _act64, _say, _t

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return _t().Generator(device=DEV).manual_seed(seed)


@pytest.mark.parametrize("m,n,width", [(1 << 20, 4100, 8), (1 << 20, 4099, 4), (70000, 65536, 4)])
def test_pack_codes_of_many(m, n, width):
    """More than 2^32 codes, more pieces than one launch has threads for."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("pack, large", m, n, width)
    codes = torch.randint(-8, 8, (m, n), dtype=torch.int8, device=DEV, generator=_gen(1))
    p = pk.pack_codes(codes, width).data
    if width == 8:
        assert torch.equal(p.view(torch.int8)[:, :n], codes)
        assert int(p[:, n:].ne(0).sum()) == 0
        return
    for rows in torch.arange(m, device=DEV).split(1 << 17):   # (temporaries of a part)
        b = p[rows[0]:rows[-1] + 1].view(len(rows), -1, 1, 4)
        got = (torch.cat((b << 4, b & 0xF0), 2).view(torch.int8) >> 4).reshape(len(rows), -1)
        assert torch.equal(got[:, :n], codes[rows[0]:rows[-1] + 1]) and int(got[:, n:].ne(0).sum()) == 0


def test_gated_mlp_pads_large_weights():
    """Odd rows, whose padded copies have more pieces than the grid that makes them has threads."""
    import paper_2608_06291_amd as pk
    torch = _t()
    T, d, f = 40, 9001, 20003
    _say("mlp, large odd weights", T, d, f)
    x, wg, wu = (torch.randn(s, device=DEV, generator=_gen(k)).mul_(c).to(torch.bfloat16)
                 for k, (s, c) in enumerate((((T, d), 1.0), ((f, d), d ** -0.5), ((f, d), d ** -0.5))))
    h = pk.gated_mlp(x, wg, wu)
    for j in (slice(0, 300), slice(f // 2, f // 2 + 300), slice(f - 300, f)):
        G, U = (x.double() @ w[j].double().t() for w in (wg, wu))
        want = _act64(G, "silu") * U
        size = x.double().abs() @ wg[j].double().abs().t()
        e = (d + 16) * U32 * (1.13 * size * U.abs() + G.abs() * (x.double().abs() @ wu[j].double().abs().t())) + 1e-6
        assert bool(((h[:, j].double() - want).abs() <= e + 2.0 ** -8 * (want.abs() + e)).all())
