"""More refusals of the operators around the cache, none of which needs a GPU."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

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


def test_binding_refuses_tensors_on_another_device(W):  # noqa: F811
    """A host pointer in a table would fault in the kernel; refused before the library sees it."""
    ctx = SimpleNamespace(index=0, handle=None)         # noqa: F811  (a context of cuda:0; these tensors are the host's)
    q, k, i, f = torch.zeros(2, 14, 64), torch.zeros(2, 2, 64), torch.zeros(2, dtype=torch.int32), torch.zeros(32)
    kv = W.PackedKV(2, 2, 64, 32, torch.float16, [0, 0, 0], [0, 4, 8], device="cpu")
    there = torch.empty(0, device="meta")               # (no device's either: any one tensor is enough)
    for call in (lambda: W.wq_rope(ctx, q, k, i, f), lambda: W.wq_rope(ctx, q, None, i, f), lambda: W.wq_rope_append_kv(ctx, q, k, k, i, f, kv),
                 lambda: W.wq_prefill_attention(ctx, q, k, k, i, i, 0.125), lambda: W.wq_decode_attention_shared(ctx, q, kv, i, None, 0.125)):
        with pytest.raises(ValueError, match="device"):
            call()
    here = SimpleNamespace(get_device=lambda: 0)
    W._here(ctx, here, None, here)
    with pytest.raises(ValueError, match="device"):
        W._here(ctx, here, None, there)


def test_more_heads_than_an_offset_of_32_bits_reaches(W, ctx):  # noqa: F811
    """2^22 fp32 heads of 128: a head lies 2^31 bytes into its row; 2^19 KV heads: a row 2^32 bytes into its tile."""
    many = 1 << 22
    assert _prefill(W, ctx, dtype=0, hd=128, Hq=many, Hkv=many // 8, qs=many * 128, tq=1, tk=0, mk=0, B=1) == -2
    assert b"heads" in W.lib().wq_last_error(ctx)
    assert _shared(W, ctx, _desc(W, B=1, Hkv=1 << 19, hd=128, group=64), B=1, Hq=1 << 19) == -2
    assert b"heads" in W.lib().wq_last_error(ctx)
    # (as many as allowed: 64 parts of each are 2^24 workgroups, past a launch's 2^32 threads; with 4 what is missing is workspace)
    assert _shared(W, ctx, _desc(W, B=1, Hkv=1 << 18, hd=128, group=64), B=1, Hq=1 << 18, splits=64) == -2
    assert b"workgroups" in W.lib().wq_last_error(ctx)
    assert _shared(W, ctx, _desc(W, B=1, Hkv=1 << 18, hd=128, group=64), B=1, Hq=1 << 18, splits=4) == -4


def test_frequencies_of_a_base_out_of_range(W):  # noqa: F811
    """10^200 stretched by 10^150^(32/30) has no place in a double; just below it has."""
    with pytest.raises(W.WQError):
        W.wq_rope_frequencies(32, 1e200, W.ROPE_BASE, 1e150)
    f = W.wq_rope_frequencies(32, 1e200, W.ROPE_BASE, 1e90)[0]           # 10^(200 + 96)
    assert all(abs(x - 10.0 ** (-296 * i / 16)) <= 2.0 ** -24 * x + 2.0 ** -149 for i, x in enumerate(f))
