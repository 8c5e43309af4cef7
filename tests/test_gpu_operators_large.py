"""GPU tests of the operators around a quantised layer at sizes whose counts and offsets pass 31 or 32 bits."""
import pytest

from test_gpu_operators import U32, _act64, _say, _slope64, _t

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


def _bf16(shape, seed, scale=1.0):
    torch = _t()
    t = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    g = _gen(seed)
    for part in t.split(max(1, (1 << 28) // shape[1])):   # (drawn in fp32, a part at a time)
        part.copy_(torch.randn(part.shape, device=DEV, generator=g).mul_(scale))
    return t


def _inside(got, want, tol, label):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (label, float((err / tol).max()))


def test_norm_beyond_32_bits():
    """More than 2^32 entries: the first and the last rows, in every output."""
    import paper_2608_06291_amd as pk
    torch = _t()
    T, d = 66000, 65536
    _say("norm, large", T, d)
    x = _bf16((T, d), 1)
    r = pk.rmsnorm_quant(x, residual=x, with_y=True)
    for rows in (slice(0, 2), slice(T // 2, T // 2 + 2), slice(T - 3, T)):
        h = 2 * x[rows].double()
        y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5)
        scale = y.abs().amax(1) / 127
        e = (d + 16) * U32
        _inside(r.sum[rows], h, 2.0 ** -8 * h.abs(), "sum")
        _inside(r.y[rows], y, (e + 2.0 ** -8 * (1 + e)) * y.abs(), "y")
        _inside(r.scale[rows], scale, e * scale, "scale")
        _inside(r.q[rows], y / scale[:, None], 0.5 + 127 * 2 * e, "q")


@pytest.mark.parametrize("T,n,m,width,group", [(34000, 65536, 70, 4, 0), (34000, 65536, 70, 8, 128),
                                               (3, 32768, 140000, 8, 0), (3, 65536, 140000, 4, 128), (90, 32768, 140000, 8, 64)])
def test_linear_reads_beyond_32_bits(T, n, m, width, group):
    """More than 2^31 bytes of rows, or 2^32 of codes: the last rows of either."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("linear, large operands", T, n, m, width, group)
    q = torch.randint(-127, 128, (T, n), dtype=torch.int8, device=DEV, generator=_gen(1))
    c = torch.randint(-7, 8, (m, n), dtype=torch.int8, device=DEV, generator=_gen(2))
    scale = torch.rand((m, n // group) if group else (m,), device=DEV, generator=_gen(3)) * 1e-3
    y = pk.linear(q, None, pk.pack_codes(c, width), scale, group_size=group, dtype=torch.float32)
    for t in (slice(0, 2), slice(T - 2, T)):
        for i in (slice(0, 40), slice(m - 40, m)):
            if group:
                p = torch.matmul(q[t].double().view(-1, n // group, group).transpose(0, 1).contiguous(),
                                 c[i].double().view(-1, n // group, group).permute(1, 2, 0).contiguous())
                p = p * scale[i].double().t()[:, None]   # group, t, i
            else:
                p = (q[t].double() @ c[i].double().t() * scale[i].double())[None]
            _inside(y[t, i], p.sum(0), (len(p) + 8) * U32 * p.abs().sum(0) + 1e-30, (t, i))


# T, d, f: more than 2^31 entries of h and dh, of x, and of the weights
LARGE = [(66000, 72, 33000), (34000, 65600, 72), (24, 65600, 33000), (80, 65601, 33000)]


@pytest.mark.parametrize("T,d,f", LARGE)
def test_gated_mlp_beyond_32_bits(T, d, f):
    import paper_2608_06291_amd as pk
    _t()
    _say("mlp, large", T, d, f)
    x, wg, wu = _bf16((T, d), 1), _bf16((f, d), 2, d ** -0.5), _bf16((f, d), 3, d ** -0.5)
    h = pk.gated_mlp(x, wg, wu)
    for t in (slice(0, 3), slice(T - 3, T)):
        for j in (slice(0, 9), slice(f - 9, f)):
            xd, a, b = x[t].double(), wg[j].double(), wu[j].double()
            G, U = xd @ a.t(), xd @ b.t()
            want = _act64(G, "silu") * U
            e = (d + 16) * U32 * (1.13 * (xd.abs() @ a.abs().t()) * U.abs() + G.abs() * (xd.abs() @ b.abs().t())) + 1e-6
            _inside(h[t, j], want, e + 2.0 ** -8 * (want.abs() + e), (t, j))


@pytest.mark.parametrize("T,d,f", LARGE)
def test_gated_mlp_backward_beyond_32_bits(T, d, f):
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("mlp backward, large", T, d, f)
    x, wg, wu = _bf16((T, d), 1), _bf16((f, d), 2, d ** -0.5), _bf16((f, d), 3, d ** -0.5)
    dh = _bf16((T, f), 4, 0.3)
    dx, dwg, dwu = pk.gated_mlp_backward(dh, x, wg, wu)

    def hidden(t, j):
        G, U = (x[t].double() @ w[j].double().t() for w in (wg, wu))
        g = dh[t, j].double()
        return g * U * _slope64(G, "silu"), g * _act64(G, "silu")

    def close(got, want, label):
        # norms: u / 2 for rounding dG and dU and u / 2 for the result's own, in bf16 (u = 2^-8), and fp32 sums
        assert float((got.double() - want).norm()) <= 0.85 * 2.0 ** -8 * float(want.norm()), label
    everything = slice(None)
    for t in (slice(0, 3), slice(T - 3, T)):
        dG, dU = hidden(t, everything)
        cols = slice(d - 64, d)
        close(dx[t, cols], dG @ wg[:, cols].double() + dU @ wu[:, cols].double(), ("dx", t))
    for j in (slice(0, 3), slice(f - 3, f)):
        dG, dU = hidden(everything, j)
        cols = slice(d - 64, d)
        close(dwg[j, cols], dG.t() @ x[:, cols].double(), ("dw_gate", j))
        close(dwu[j, cols], dU.t() @ x[:, cols].double(), ("dw_up", j))


def test_operators_from_two_threads():
    """Two threads, each on a stream of its own, with operators that take workspaces: the same bits as alone."""
    import threading

    import paper_2608_06291_amd as pk
    torch = _t()
    _say("threads")

    def inputs(k):
        T, d, f = (40, 333, 200) if k else (300, 264, 1000)
        return (_bf16((T, d), k), _bf16((f, d), k + 10, d ** -0.5), _bf16((f, d), k + 20, d ** -0.5), _bf16((T, f), k + 30),
                torch.randn((2 + k, 70000), device=DEV, generator=_gen(k)))

    def work(x, wg, wu, dh, z):
        n = pk.rmsnorm_quant(x, with_y=True)
        lp = pk.token_logprobs(z, None, top=9)
        return [n.q.contiguous(), n.scale, pk.gated_mlp(n.y, wg, wu), *pk.gated_mlp_backward(dh, x, wg, wu), lp.lse, lp.top_index,
                pk.token_logprobs_backward(z, None, lp.lse, lp.entropy, g_entropy=lp.lse)]
    args = [inputs(k) for k in range(2)]
    want = [[t.clone() for t in work(*a)] for a in args]
    torch.cuda.synchronize()
    wrong = []

    def run(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for i in range(30):
                    got = work(*args[k])
                    st.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                        wrong.append((k, i))
        except Exception as e:   # (seen by the test, not lost with the thread)
            wrong.append((k, repr(e)))
    threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not wrong and not any(t.is_alive() for t in threads), wrong[:4]
