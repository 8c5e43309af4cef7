"""GPU tests of how the operators at the ends of a network may be called: captured into graphs, from threads, on other
streams, with workspaces, tensors that require gradients, views, rows beyond 32-bit offsets, special values."""
import math
import threading

import pytest

from test_gpu_network_ends import DEV, U32, _head_inputs, _rand, _say, _t, _tokens

pytestmark = pytest.mark.gpu


def _inputs(T, d, V, dtype="bf16", seed=0):
    torch = _t()
    x, w, tok = (t.to(DEV) for t in _head_inputs(T, d, V, dtype, seed))
    weight, bias = (torch.randn(d, device=DEV, generator=torch.Generator(DEV).manual_seed(seed + k)) for k in (5, 6))
    gl = -torch.rand((T,), device=DEV, generator=torch.Generator(DEV).manual_seed(seed + 7)) / T
    return x, w, tok, weight, bias, gl


def _all(x, w, tok, weight, bias, gl):
    """Every operator, as they are used together."""
    import paper_2608_06291_amd as pk
    V = w.shape[0]
    e = pk.embedding(tok, w, scale=2.0)
    n = pk.layernorm(e, weight, bias, residual=x)
    r = pk.layernorm(n.sum, weight, centre=False)
    lp = pk.head_logprobs(r.y, w, tok)
    dr, dw = pk.head_logprobs_backward(r.y, w, tok, lp.lse, lp.entropy, gl, gl)
    dsum, dweight, _ = pk.layernorm_backward(dr, n.sum, weight, None, r.rstd)
    dx, dweight2, dbias = pk.layernorm_backward(dr, n.sum, weight, n.mean, n.rstd, d_sum=dsum)
    dw2 = pk.embedding_backward(dx, tok, V, scale=2.0, base=dw)
    return [e, n.y, n.mean, n.rstd, n.sum, r.y, *lp[:3], dr, dw, dsum, dweight, dx, dweight2, dbias, dw2]


@pytest.mark.parametrize("T,d,V,dtype", [(1, 96, 500, "bf16"), (30, 131, 3000, "f16"), (300, 264, 9000, "f16"), (1000, 520, 9000, "bf16")])
def test_captured_and_replayed(T, d, V, dtype):
    """A graph of all of them, replayed with eager calls between the replays, on other inputs in the same places."""
    torch = _t()
    _say("graph", T, d, V, dtype)
    args = _inputs(T, d, V, dtype)
    _all(*args)
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        out = _all(*args)
    for seed in (0, 100, 200, 0):
        for a, b in zip(args, _inputs(T, d, V, dtype, seed)):
            a.copy_(b)
        want = [t.clone() for t in _all(*args)]
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), (seed, i)


def test_two_graphs_with_workspaces():
    """Two captured calls, each with a workspace of its own, replayed at once on two streams."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("two graphs")
    args = [_inputs(200 + 70 * k, 264, 5000, seed=k) for k in range(2)]
    lse = [pk.head_logprobs(a[0], a[1]).lse for a in args]
    calls = [lambda k=k, work=None: pk.head_logprobs_backward(args[k][0], args[k][1], args[k][2], lse[k], g_logprob=args[k][5], work=work)
             for k in range(2)]
    want = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], []
    works = [torch.empty(1 << 27, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for k in range(2):
        streams.append(torch.cuda.Stream())
        graphs.append(torch.cuda.CUDAGraph())
        streams[k].wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graphs[k], stream=streams[k]):
            outs.append(calls[k](work=works[k]))
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))


def test_two_threads():
    torch = _t()
    _say("threads")
    args = [_inputs(300, 264, 3000, "f16"), _inputs(20, 131, 5000, "bf16", 9)]
    want = [[t.clone() for t in _all(*a)] for a in args]
    torch.cuda.synchronize()
    wrong = []

    def run(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for i in range(20):
                    got = _all(*args[k])
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


def test_tensors_that_require_gradients_are_refused():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("requires_grad")
    x, w, tok, weight, bias, _ = _inputs(5, 64, 90)
    for call, tensors in ((lambda: pk.head_logprobs(x, w, tok), (x, w)), (lambda: pk.layernorm(x, weight, bias, x), (x, weight, bias)),
                          (lambda: pk.embedding(tok, w), (w,))):
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


def test_what_the_binding_refuses():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("refusals")
    x, w, tok, weight, bias, gl = _inputs(5, 64, 90)
    lse = gl.clone()
    bad = [lambda: pk.head_logprobs(x, w[:, :63], tok), lambda: pk.head_logprobs(x, w.half(), tok), lambda: pk.head_logprobs(x.float(), w.float(), tok),
           lambda: pk.head_logprobs(x, w, tok[:4]), lambda: pk.head_logprobs(x, w, tok.int()), lambda: pk.head_logprobs(x, w.t(), tok),
           lambda: pk.head_logprobs(x[0], w, tok), lambda: pk.head_logprobs(x, w, tok, work=torch.empty(1 << 20)),
           lambda: pk.head_logprobs(x, w, tok, work=torch.empty(16, dtype=torch.uint8, device=DEV)),
           lambda: pk.head_logprobs_backward(x, w, tok, lse.double(), g_logprob=gl),
           lambda: pk.head_logprobs_backward(x, w, None, lse, g_logprob=gl), lambda: pk.head_logprobs_backward(x, w, tok, lse, g_entropy=gl),
           lambda: pk.head_logprobs_backward(x, w, tok, lse, need_dx=False, need_dw=False),
           lambda: pk.layernorm(x, weight[:63]), lambda: pk.layernorm(x, weight.half()), lambda: pk.layernorm(x, residual=x.half()),
           lambda: pk.layernorm(x, residual=x[:4]), lambda: pk.layernorm(x, eps=0.0), lambda: pk.layernorm(x.t()), lambda: pk.layernorm(x.double()),
           lambda: pk.layernorm(x, sum_out=x.float()), lambda: pk.layernorm_backward(x, x, weight, lse[:4], lse),
           lambda: pk.layernorm_backward(x, x[:, :8], weight, None, lse), lambda: pk.layernorm_backward(x, x, weight, None, lse, d_sum=x.float()),
           lambda: pk.layernorm_backward(x, x, weight, None, lse, need_dx=False, need_dweight=False, need_dbias=False),
           lambda: pk.embedding(tok[None], w), lambda: pk.embedding(tok.int(), w), lambda: pk.embedding(tok, w.long()),
           lambda: pk.embedding(tok[::2], w), lambda: pk.embedding(tok, w, out=x.float()), lambda: pk.embedding(tok.cpu(), w),
           lambda: pk.embedding_backward(x, tok[:3], 90), lambda: pk.embedding_backward(x, tok, 0),
           lambda: pk.embedding_backward(x, tok, 90, base=w[:80]), lambda: pk.embedding_backward(x, tok, 90, out=w.float()),
           lambda: pk.embedding_backward(x.long(), tok, 90)]
    for k, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError, pk.BakronError)):
            call()
            pytest.fail(f"call {k} was taken")


def test_empty_calls():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("T = 0")
    x, w, tok, weight, bias, gl = _inputs(5, 64, 90)
    x0, t0, f0 = x[:0], tok[:0], gl[:0]
    lp = pk.head_logprobs(x0, w, t0)
    assert lp.logprob.shape == lp.lse.shape == lp.entropy.shape == (0,)
    dx, dw = pk.head_logprobs_backward(x0, w, t0, f0, g_logprob=f0)
    assert dx.shape == (0, 64) and dw.shape == w.shape and not bool(dw.any())
    n = pk.layernorm(x0, weight, bias, residual=x0)
    assert n.y.shape == n.sum.shape == (0, 64) and n.mean.shape == (0,)
    dx, dweight, dbias = pk.layernorm_backward(x0, x0, weight, f0, f0)
    assert dx.shape == (0, 64) and not bool(dweight.any()) and not bool(dbias.any())
    assert pk.embedding(t0, w).shape == (0, 64)
    assert not bool(pk.embedding_backward(x0, t0, 90).any())


@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T", (6, 40, 300))
def test_head_special_rows(dtype, T):
    """Logits that are NaN or infinite: their rows alone, and rows behind the outputs left as they were."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head special", dtype, T)
    x, w, tok, _, _, gl = _inputs(T, 96, 700, dtype)
    want = pk.head_logprobs(x, w, tok)
    g0 = pk.head_logprobs_backward(x, w, tok, want.lse, want.entropy, gl, gl, need_dw=False)[0]
    bad = x.clone()
    bad[0, 3], bad[2, 95], bad[4, 0] = math.nan, math.inf, -math.inf
    got = pk.head_logprobs(bad, w, tok)
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[[0, 2, 4]] = False
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a[keep], b[keep])
    assert bool(torch.isnan(got.lse[~keep]).all()) and bool(torch.isnan(got.entropy[~keep]).all())
    asked = (tok >= 0) & (tok < 700)
    assert torch.equal(torch.isnan(got.logprob), ~keep & asked)
    dx = pk.head_logprobs_backward(bad, w, tok, got.lse, got.entropy, gl, gl, need_dw=False)[0]
    assert torch.equal(dx[keep], g0[keep]) and bool(torch.isnan(dx[~keep]).all())
    # rows whose logits are all -inf, by their statistics: nothing comes back
    lse, H = want.lse.clone(), want.entropy.clone()
    lse[1], H[1] = -math.inf, 0.0
    dx, dw = pk.head_logprobs_backward(x, w, tok, lse, H, gl, gl)
    assert not bool(dx[1].any()) and torch.equal(dx[keep][1:], g0[keep][1:]) and bool(torch.isfinite(dw).all())
    # tokens that ask for nothing give nothing
    none = torch.full((T,), -1, device=DEV)
    dx, dw = pk.head_logprobs_backward(x, w, none, want.lse, g_logprob=gl)
    assert not bool(dx.any()) and not bool(dw.any())
    assert not bool(pk.head_logprobs(x, w, none).logprob.any())


def test_half_precision_gradients_of_any_size():
    """Gradients far below what half precision holds, and up to its largest number, lose no bits on the way to dx."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head, range")
    for T in (20, 200):
        x, w, tok, _, _, gl = _inputs(T, 256, 900, "f16")
        x = x / 16
        lp = pk.head_logprobs(x, w, tok)
        base = pk.head_logprobs_backward(x, w, tok, lp.lse, g_logprob=gl)
        for e in (-8, 6):   # a power of two throughout: the same numbers, but for what underflows in the results
            got = pk.head_logprobs_backward(x, w, tok, lp.lse, g_logprob=gl * 2.0 ** e)
            for a, b in zip(got, base):
                far = (a.double() * 2.0 ** -e - b.double()).abs()
                assert bool((far <= 2.0 ** -24 * (2.0 ** -e + 1)).all()), (T, e)


def test_outputs_leave_the_rest_alone():
    """Rows of wider buffers: what lies between and behind them stays as it was (through the C entries)."""
    import ctypes

    import paper_2608_06291_amd as pk
    torch = _t()
    _say("bounds")
    lib = pk.load()
    st = torch.cuda.current_stream().cuda_stream
    for T, d, V in ((3, 67, 100), (40, 130, 333), (300, 72, 700), (600, 200, 9001)):
        x, w, tok, weight, bias, gl = _inputs(T, d, V)
        lp = pk.head_logprobs(x, w, tok)
        want = pk.head_logprobs_backward(x, w, tok, lp.lse, g_logprob=gl)
        dx, dw = (torch.full((n + 1, d + 5), 9.0, dtype=x.dtype, device=DEV) for n in (T, V))
        size = ctypes.c_size_t(0)
        args = [x.data_ptr(), d, T, d, w.data_ptr(), d, V, 2, tok.data_ptr(), lp.lse.data_ptr(), None, gl.data_ptr(), None, dx.data_ptr(), d + 5,
                dw.data_ptr(), d + 5]
        assert lib.bakron_head_logprobs_backward(*args, None, ctypes.byref(size), st) == 0
        work = torch.full((size.value + 4096,), 170, dtype=torch.uint8, device=DEV)
        assert lib.bakron_head_logprobs_backward(*args, work.data_ptr(), ctypes.byref(size), st) == 0
        torch.cuda.synchronize()
        assert bool((work[size.value:] == 170).all())
        for got, a, n in zip((dx, dw), want, (T, V)):
            assert torch.equal(got[:n, :d], a) and bool((got[:, d:] == 9).all()) and bool((got[n] == 9).all())
        args = [x.data_ptr(), d, T, d, w.data_ptr(), d, V, 2, tok.data_ptr()]
        stats = torch.full((3, T + 4), 9.0, device=DEV)
        out = [stats[k].data_ptr() for k in range(3)]
        assert lib.bakron_head_logprobs(*args, *out, None, ctypes.byref(size), st) == 0
        work = torch.full((size.value + 4096,), 170, dtype=torch.uint8, device=DEV)
        assert lib.bakron_head_logprobs(*args, *out, work.data_ptr(), ctypes.byref(size), st) == 0
        torch.cuda.synchronize()
        assert bool((work[size.value:] == 170).all()) and bool((stats[:, T:] == 9).all())
        assert all(torch.equal(stats[k, :T], lp[k]) for k in range(3))
        # embedding: gradient, workspace
        table = torch.full((V + 1, d + 5), 9.0, dtype=x.dtype, device=DEV)
        args = [x.data_ptr(), d, tok.data_ptr(), T, 2, V, d, 1.0, None, d, table.data_ptr(), d + 5]
        assert lib.bakron_embedding_backward(*args, None, ctypes.byref(size), st) == 0
        work = torch.full((size.value + 4096,), 170, dtype=torch.uint8, device=DEV)
        assert lib.bakron_embedding_backward(*args, work.data_ptr(), ctypes.byref(size), st) == 0
        torch.cuda.synchronize()
        assert bool((work[size.value:] == 170).all())
        assert torch.equal(table[:V, :d], pk.embedding_backward(x, tok, V)) and bool((table[:, d:] == 9).all()) and bool((table[V] == 9).all())
        # norm: outputs, workspace
        n = pk.layernorm(x, weight, bias)
        dx = torch.full((T + 1, d + 5), 9.0, dtype=x.dtype, device=DEV)
        dwb = torch.full((2, d + 7), 9.0, device=DEV)
        args = [x.data_ptr(), d, x.data_ptr(), d, 2, T, d, weight.data_ptr(), n.mean.data_ptr(), n.rstd.data_ptr(), None, d, dx.data_ptr(), d + 5,
                dwb[0].data_ptr(), dwb[1].data_ptr()]
        assert lib.bakron_layernorm_backward(*args, None, ctypes.byref(size), st) == 0
        work = torch.full((size.value + 4096,), 170, dtype=torch.uint8, device=DEV)
        assert lib.bakron_layernorm_backward(*args, work.data_ptr(), ctypes.byref(size), st) == 0
        torch.cuda.synchronize()
        want = pk.layernorm_backward(x, x, weight, n.mean, n.rstd)
        assert bool((work[size.value:] == 170).all()) and bool((dx[:, d:] == 9).all()) and bool((dx[T] == 9).all()) and bool((dwb[:, d:] == 9).all())
        assert torch.equal(dx[:T, :d], want[0]) and torch.equal(dwb[0, :d], want[1]) and torch.equal(dwb[1, :d], want[2])


def test_in_place():
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("in place")
    for T, d in ((5, 64), (300, 1001), (40, 20000)):
        x, r = (_rand((T, d), k).to(torch.bfloat16).to(DEV) for k in (1, 2))
        want = pk.layernorm(x, residual=r)
        mine = r.clone()
        got = pk.layernorm(x, residual=mine, sum_out=mine)
        assert torch.equal(got.y, want.y) and torch.equal(mine, want.sum) and got.sum.data_ptr() == mine.data_ptr()
        mine = x.clone()
        got = pk.layernorm(mine, residual=r, sum_out=mine)
        assert torch.equal(got.y, want.y) and torch.equal(mine, want.sum)


@pytest.mark.parametrize("T", [16384, 16385, 20000, 300000])
def test_sorts_of_many_tokens(T):
    """Both ways of sorting, at their border and with one token throughout, against sums by index in 64 bits."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("sort", T)
    d = 24
    dy = _rand((T, d), 1).to(torch.float32)
    for V, tok in ((1 << 20, torch.randint(0, 1 << 20, (T,), generator=torch.Generator().manual_seed(1))), (3000, _tokens(T, 3000, 2)),
                   (5, torch.full((T,), 3)), (2049, torch.randint(0, 2049, (T,), generator=torch.Generator().manual_seed(3)))):
        got = pk.embedding_backward(dy.to(DEV), tok.to(DEV), V).cpu().double()
        ok = (tok >= 0) & (tok < V)
        want, size = (torch.zeros((V, d), dtype=torch.float64).index_add_(0, tok[ok], v[ok].double()) for v in (dy, dy.abs()))
        n = torch.bincount(tok[ok], minlength=V)[:, None]
        assert bool(((got - want).abs() <= (n + 2) * U32 * size).all()), V


def _bf16(shape, seed, scale=1.0):
    torch = _t()
    t = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(seed)
    for part in t.split(max(1, (1 << 28) // shape[1])):   # (drawn in fp32, a part at a time)
        part.copy_(torch.randn(part.shape, device=DEV, generator=g).mul_(scale))
    return t


def test_norm_beyond_32_bits():
    """More than 2^32 entries: the first and the last rows, and the columns' sums."""
    import paper_2608_06291_amd as pk
    torch = _t()
    for T, d in ((66000, 65536), (600000, 8192)):
        _say("norm, large", T, d)
        x = _bf16((T, d), 1)
        n = pk.layernorm(x, residual=x)
        f = pk.layernorm_backward(n.y, n.sum, None, n.mean, n.rstd, d_sum=x)
        for rows in (slice(0, 2), slice(T // 2, T // 2 + 2), slice(T - 3, T)):
            h = n.sum[rows].double()
            assert bool(((h - 2 * x[rows].double()).abs() <= 2.0 ** -8 * 2 * x[rows].double().abs()).all())
            m = h.mean(1, keepdim=True)
            y = (h - m) / torch.sqrt((h - m).square().mean(1, keepdim=True) + 1e-5)
            e = (d + 16) * U32
            assert bool(((n.y[rows].double() - y).abs() <= 2.0 ** -8 * y.abs() + e * (1 + y.abs())).all())
            g, r = n.y[rows].double(), n.rstd[rows].double()[:, None]
            dx = (g - g.mean(1, keepdim=True) - y * (g * y).mean(1, keepdim=True)) * r + x[rows].double()
            assert bool(((f[0][rows].double() - dx).abs() <= 2.0 ** -8 * dx.abs() + 4 * e * (1 + y.abs() + x[rows].double().abs())).all())
        part = n.y[:, -64:].double()
        assert bool(((f[2][-64:].double() - part.sum(0)).abs() <= (T + 2) * U32 * part.abs().sum(0)).all())
        del x, n, f, part


def test_embedding_beyond_32_bits():
    import paper_2608_06291_amd as pk
    torch = _t()
    V, d, T = 70000, 65536, 66000
    _say("embedding, large")
    table = _bf16((V, d), 1)
    tok = torch.arange(V - T, V, device=DEV)
    y = pk.embedding(tok, table)
    for rows in (slice(0, 2), slice(T - 2, T)):
        assert torch.equal(y[rows], table[tok[rows]])
    g = pk.embedding_backward(y, tok, V, base=table)
    want = torch.cat([table[:2].float(), 2 * table[-2:].float()]).to(torch.bfloat16)
    assert torch.equal(torch.cat([g[:2], g[-2:]]), want)


@pytest.mark.parametrize("T,d,V", [(34000, 65600, 72), (70, 65600, 33000), (20, 65600, 33000), (40000, 64, 120000)])
def test_head_beyond_32_bits(T, d, V):
    """More than 2^31 entries of x, of w, of the gradients, and of the logits that are not kept."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head, large", T, d, V)
    x, w = _bf16((T, d), 1), _bf16((V, d), 2, d ** -0.5)
    tok = torch.arange(T, device=DEV) % V
    lp = pk.head_logprobs(x, w, tok)
    gl = torch.full((T,), -1.0, device=DEV)
    dx, dw = pk.head_logprobs_backward(x, w, tok, lp.lse, g_logprob=gl)

    def dz(t, part=slice(None)):
        z = x[t].double() @ w.double().t() if V * d < 1 << 29 else torch.cat([x[t].double() @ p.double().t() for p in w.split(4096)], 1)
        p = torch.softmax(z, 1)
        p[torch.arange(len(p)), tok[t]] -= 1
        return z, p
    for t in (slice(0, 3), slice(T - 3, T)):
        z, p = dz(t)
        lse = torch.logsumexp(z, 1)
        e = 2 * (d + 1) * U32 * 6 + V * U32
        assert bool(((lp.lse[t].double() - lse).abs() <= e * (1 + lse.abs())).all())
        cols = slice(d - 64, d)
        want = p @ w[:, cols].double()
        # norms: u / 2 for rounding dz and u / 2 for the result's own (u = 2^-8), and fp32 sums
        assert float((dx[t, cols].double() - want).norm()) <= 0.85 * 2.0 ** -8 * float(want.norm()), t
    for v in (slice(0, 3), slice(V - 3, V)):
        z = torch.cat([a.double() @ w[v].double().t() for a in x.split(1 << 13)])
        p = torch.exp(z - lp.lse.double()[:, None]) - (tok[:, None] == torch.arange(V, device=DEV)[v][None]).double()
        want = p.t().contiguous() @ x[:, d - 64:].double()
        assert float((dw[v, d - 64:].double() - want).norm()) <= 0.85 * 2.0 ** -8 * float(want.norm()), v


def test_workspaces_of_calls_that_differ_in_alignment_only():
    """The binding keeps the sizes that it has asked for: rows that have to be copied need more."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("kept sizes")
    T, d, V = 100, 128, 3000
    x, w, tok, _, _, gl = _inputs(T, d, V)
    want = pk.head_logprobs(x, w, tok)
    grads = pk.head_logprobs_backward(x, w, tok, want.lse, g_logprob=gl)
    for px, pw in ((0, 1), (1, 0), (8, 8), (3, 3), (0, 0)):
        xs, ws = (torch.empty((n, d + p), dtype=x.dtype, device=DEV)[:, p // 2:p // 2 + d] for n, p in ((T, px), (V, pw)))
        xs.copy_(x), ws.copy_(w)
        assert all(torch.equal(a, b) for a, b in zip(pk.head_logprobs(xs, ws, tok)[:3], want[:3]))
        got = pk.head_logprobs_backward(xs, ws, tok, want.lse, g_logprob=gl)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
