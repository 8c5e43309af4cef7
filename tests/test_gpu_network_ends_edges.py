"""GPU tests of the operators at the ends of a network where calls of one kind meet inputs of another: rows that ask for
nothing beside rows that do, results in the place of inputs, statistics that have to be better than a bound of the worst
case says."""
import math

import pytest

from network_ends_sizes import HEAD, HEAD_LARGE
from test_gpu_network_ends import DEV, U32, _dtype, _head_inputs, _rand, _say, _strided, _t, _tiny, _u

pytestmark = pytest.mark.gpu


# every place that the scale of half precision is taken in: up to 16 and 32 rows, few rows of few tokens, 65 to 512 rows
# in tiles, more; each with one and two results
@pytest.mark.parametrize("dtype", ("f16", "bf16"))
@pytest.mark.parametrize("T,d,V", [(5, 256, 900), (20, 256, 900), (6, 5, 900), (40, 256, 900), (40, 520, 300), (200, 256, 900), (600, 256, 900)])
def test_rows_that_ask_for_nothing_do_not_scale(dtype, T, d, V):
    """Whatever comes in at a row without a target, or without a finite logit, changes nothing of the others."""
    import paper_2608_06291_amd as pk
    torch = _t()
    _say("head, rows without a target", dtype, T, d, V)
    x, w, tok = (t.to(DEV) for t in _head_inputs(T, d, V, dtype))
    lp = pk.head_logprobs(x, w, tok)
    lse, H = lp.lse.clone(), lp.entropy.clone()
    tok[1], tok[T - 1], tok[2] = -100, V, V // 3
    lse[2], H[2] = -math.inf, 0.0        # logits of -inf throughout
    g = torch.Generator().manual_seed(3)
    gl, gh = (((torch.rand((T,), generator=g) - 0.5) / T).to(DEV) for _ in range(2))
    nothing = (tok < 0) | (tok >= V)
    for entropy in (False, True):
        want = None
        for size in (0.0, 1e30, -1e4, 3e38):
            a, b = gl.clone(), gh.clone()
            a[nothing] = size
            a[2] = b[2] = size
            args = (x, w, tok, lse, H if entropy else None, a, b if entropy else None)
            got = pk.head_logprobs_backward(*args)
            want = got if want is None else want
            assert bool(want[0][0].any()) and bool(want[1].any())
            for p, q in zip(got, want):
                assert torch.equal(p, q), (entropy, size)
            assert torch.equal(pk.head_logprobs_backward(*args, need_dw=False)[0], want[0])
            assert torch.equal(pk.head_logprobs_backward(*args, need_dx=False)[1], want[1])
    # without gradients of log probabilities the targets ask for nothing either way
    got = [pk.head_logprobs_backward(x, w, t, lse, H, None, gh) for t in (tok, None)]
    assert all(torch.equal(p, q) for p, q in zip(*got))
