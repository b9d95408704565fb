"""More refusals of the operators around the cache, none of which needs a GPU."""
import ctypes as C

import pytest

from tests.test_operators_host import BF, P, W, _desc, _prefill, _rope, ctx  # noqa: F401


def _shared(W, ctx, prefix, own=None, **more):  # noqa: F811
    a = dict(B=2, Hq=14, sm=0.125, splits=1)
    a.update(more)
    return W.lib().wq_decode_attention_shared(ctx, P, BF, a["B"], a["Hq"], C.byref(prefix), P, None if own is None else C.byref(own), a["sm"], a["splits"], 100, 100,
                                              P, None)


@pytest.mark.parametrize("sm,code", [(2.9e38, -1), (2.4e38, -1), (2.3e38, -4), (1e-45, -4), (1e-46, -1)])
def test_scales_at_the_ends_of_fp32(W, ctx, sm, code):  # noqa: F811
    """Exponents are powers of two: the scale times log2(e) has to be finite.  (-4: accepted, and then too little workspace.)"""
    assert _prefill(W, ctx, sm=sm, tq=1000000, splits=2) == code
    assert _shared(W, ctx, _desc(W), sm=sm, B=1000, splits=64) == code
