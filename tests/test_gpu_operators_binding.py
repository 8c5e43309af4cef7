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


def test_pack_refuses_codes_that_do_not_fit():
    """4 bits hold -8 .. 7: what is beyond would lose its upper bits."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("pack, range")
    for bad in (8, -9, 127, -128):
        codes = torch.zeros((3, 40), dtype=torch.int8, device=DEV)
        codes[2, 39] = bad
        with pytest.raises(ValueError):
            pk.pack_codes(codes)
        assert pk.pack_codes(codes, check=False).data.shape == (3, 64)
        assert int(pk.pack_codes(codes, 8).data.view(torch.int8)[2, 39]) == bad
    codes[2, 38:] = torch.tensor([-8, 7], dtype=torch.int8)
    assert int(pk.pack_codes(codes).data[2, 18]) == 0x80 and int(pk.pack_codes(codes).data[2, 19]) == 0x70
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()   # a capture cannot wait, and is not made to
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        p = pk.pack_codes(codes)
    g.replay()
    assert torch.equal(p.data, pk.pack_codes(codes).data)


def test_workspaces_have_to_be_device_memory():
    """Kernels write to a workspace: host memory, or a tensor with gaps, is refused before any work."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("workspaces")
    bf = dict(dtype=torch.bfloat16, device=DEV)
    x, w, z = torch.zeros((70, 65), **bf), torch.zeros((300, 65), **bf), torch.zeros((1, 60000), device=DEV)
    q, _, packed = _layer()
    for work in (torch.empty(1 << 24, dtype=torch.uint8), torch.empty((1 << 12, 1 << 13), dtype=torch.uint8, device=DEV)[:, ::2]):
        for call in (lambda: pk.gated_mlp(x, w, w, work=work), lambda: pk.token_logprobs(z, work=work),
                     lambda: pk.gated_mlp_backward(torch.zeros((70, 300), **bf), x, w, w, work=work),
                     lambda: pk.linear(q, None, packed, torch.ones(6, device=DEV), work=work),
                     lambda: pk.gram(x.float(), work=work)):
            with pytest.raises(ValueError):
                call()
    good = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    assert torch.equal(pk.gated_mlp(x, w, w, work=good), pk.gated_mlp(x, w, w))


def test_linear_takes_packed_bytes_only():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("packed bytes")
    q, _, w = _layer()
    one = torch.ones(6, device=DEV)
    for data in (w.data.float(), w.data.to(torch.int16), w.data.cpu(), w.data[:, ::2], w.data[:, :64]):
        with pytest.raises(ValueError):
            pk.linear(q, None, w._replace(data=data), one)


def test_calls_that_would_lose_gradients_are_refused():
    """The operators record no graph: with a tensor that asks for one they raise, they do not detach."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("graphs")
    q, _, w = _layer()
    bf = dict(dtype=torch.bfloat16, device=DEV)

    def rand(*shape, **kw):
        return torch.randn(shape, **(kw or bf))
    x, wg, wu, z = rand(3, 64), rand(40, 64), rand(40, 64), rand(3, 500)
    f32 = dict(device=DEV)
    norm, scale, qs, bias, other = rand(64, **f32), rand(6, **f32), rand(3, **f32), rand(6), rand(3, 6)
    calls = [(lambda: pk.rmsnorm_quant(x, norm, x), (x, norm)), (lambda: pk.gated_mlp(x, wg, wu), (x, wg, wu)),
             (lambda: pk.linear(q, qs, w, scale, bias=bias, other=other), (qs, scale, bias, other)),
             (lambda: pk.token_logprobs(z), (z,))]
    for call, tensors in calls:
        want = call()
        for t in tensors:
            t.requires_grad_(True)
            with pytest.raises(RuntimeError, match="no_grad"):
                call()
            with torch.no_grad():
                got = call()
            t.requires_grad_(False)
            for a, b in zip(*((v,) if isinstance(v, torch.Tensor) else v for v in (got, want))):
                assert (a is None and b is None) or torch.equal(a, b)
    # gradients as values, of parameters too
    wg.requires_grad_(True)
    assert all(not g.requires_grad for g in pk.gated_mlp_backward(rand(3, 40), x, wg, wu))


def test_gated_mlp_of_one_feature_takes_any_distance():
    """One row has no next one: views whose rows would lie at different distances are the same weights."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("one feature")
    bf = dict(dtype=torch.bfloat16, device=DEV)
    x, wide, dh = torch.randn((5, 64), **bf), torch.randn((3, 160), **bf), torch.randn((5, 1), **bf)
    wg, wu = torch.randn((1, 64), **bf), wide[1:2, 8:72]
    want = pk.gated_mlp(x, wg, wu.clone())
    assert torch.equal(pk.gated_mlp(x, wg, wu), want) and torch.equal(pk.gated_mlp(x, wg, wide[::2][1:, 8:72]),
                                                                      pk.gated_mlp(x, wg, wide[2:, 8:72].clone()))
    for a, b in zip(pk.gated_mlp_backward(dh, x, wg, wu), pk.gated_mlp_backward(dh, x, wg, wu.clone())):
        assert torch.equal(a, b)
