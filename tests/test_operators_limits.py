"""Numbers of rows that the operators around a quantised layer refuse, up to the largest that an
argument holds: needs no GPU (the pointers are never followed)."""
import ctypes

import pytest

from test_operators_refusals import (BWD, BWD_OK, LINEAR, LINEAR_OK, LP, LP_OK, LPB, LPB_OK, MLP, MLP_OK, NORM, NORM_OK,
                                     _call, _size, lib)  # noqa: F401

CALLS = {"bakron_rmsnorm_quant": (NORM, NORM_OK), "bakron_linear": (LINEAR, LINEAR_OK), "bakron_gated_mlp": (MLP, MLP_OK),
         "bakron_gated_mlp_backward": (BWD, BWD_OK), "bakron_token_logprobs": (LP, LP_OK),
         "bakron_token_logprobs_backward": (LPB, LPB_OK)}


@pytest.mark.parametrize("T", [1 << 31, (1 << 32) + 1, (1 << 62) + 3, (1 << 63) - 64, (1 << 63) - 1, -(1 << 63)])
@pytest.mark.parametrize("name", CALLS)
def test_rows_beyond_the_limit(lib, name, T):  # noqa: F811
    names, base = CALLS[name]
    if "work" in names:   # asking for the workspace is refused, too
        base = dict(base, size=_size(0), work=None)
    assert _call(getattr(lib, name), names, base, T=T) == 1
    assert name.encode() in lib.bakron_last_error()
    if "work" in names:
        need = ctypes.c_size_t(77)
        _call(getattr(lib, name), names, dict(base, size=ctypes.byref(need)), T=T)
        assert need.value == 77


@pytest.mark.parametrize("name", ["bakron_gated_mlp", "bakron_gated_mlp_backward"])
def test_rows_whose_launch_passes_64_bits(lib, name):  # noqa: F811
    """At the widest layer 8193 workgroups take 64 rows: so many rows that their product wraps around to
    a small number."""
    names, base = CALLS[name]
    wide = 1 << 17
    blocks = -(-(1 << 64) // 8193)
    assert blocks * 8193 % (1 << 64) < 8193
    base = dict(base, size=_size(0), work=None, d=wide, f=wide,
                **{n: 1 << 18 for n in ("ldx", "ldw", "ldh", "lddh", "lddx", "lddw") if n in names})
    assert _call(getattr(lib, name), names, base, T=100) == 0
    assert _call(getattr(lib, name), names, base, T=blocks * 64) == 1
