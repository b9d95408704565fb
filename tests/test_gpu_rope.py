"""Rotary positions against their definition in 64 bits, and the append form against the two calls that it stands for."""
import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _inputs(rows, Hq, Hkv, hd, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(rows, (Hq + 2 * Hkv) * hd, generator=g) * spread).to(dtype).cuda()
    cut = lambda a, z: qkv[:, a * hd:z * hd].unflatten(-1, (-1, hd))  # noqa: E731
    return cut(0, Hq), cut(Hq, Hq + Hkv), cut(Hq + Hkv, Hq + 2 * Hkv)


def _close(got, x, positions, inv_freq, layout, mscale):
    """One rounding to the type; before it fp32: the reduced angle is a fp32 number of half turns up to 1 (its rounding is 2^-25 pi), cosine and
    sine, their factor, two products and their sum are off by a step of 2^-24 or two each: below 8 * 2^-24 of the two terms' magnitudes."""
    want, size = R.rope(x.double().cpu(), positions.cpu(), inv_freq.cpu(), layout, mscale)
    bound = R.HALF_STEP[got.dtype] * want.abs() + 8 * 2.0 ** -24 * size + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    rot = 2 * inv_freq.numel()
    assert torch.equal(got[..., rot:], x[..., rot:]), "channels behind rot_dim"
    assert bool(((got.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", [W.ROPE_HALF, W.ROPE_PAIRS])
@pytest.mark.parametrize("rows,Hq,Hkv,hd,rot", [(1, 1, 1, 64, 64), (3, 14, 2, 64, 32), (5, 28, 4, 128, 128), (130, 7, 1, 128, 96), (67, 8, 8, 64, 16)])
def test_rows(dtype, layout, rows, Hq, Hkv, hd, rot):
    q, k, _ = _inputs(rows, Hq, Hkv, hd, dtype, rows + rot)
    g = torch.Generator().manual_seed(rot)
    positions = torch.randint(-2000000, 2000000, (rows,), generator=g, dtype=torch.int32).cuda()
    positions[0] = 0 if rows > 1 else 2 ** 31 - 1
    f, m = W.wq_rope_frequencies(rot, 10000.0, W.ROPE_PARTS, 4.0, 8192)
    inv_freq = torch.tensor(f).cuda()
    ctx = W.Context(0)
    qo, ko = W.wq_rope(ctx, q, k, positions, inv_freq, layout, m)
    _close(qo, q, positions, inv_freq, layout, m)
    _close(ko, k, positions, inv_freq, layout, m)
    # queries alone; in place in the fused rows, whose values stay
    q1, none = W.wq_rope(ctx, q, None, positions, inv_freq, layout, m)
    assert none is None and torch.equal(q1, qo)
    q2, k2, v2 = _inputs(rows, Hq, Hkv, hd, dtype, rows + rot)
    before = v2.clone()
    W.wq_rope(ctx, q2, k2, positions, inv_freq, layout, m, q_out=q2, k_out=k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko) and torch.equal(v2, before)


def test_more_rows_than_a_launch_takes():
    """2^26 - 4 rows fill a launch of 2^24 - 1 workgroups; in place, one head, 8.6 GB."""
    rows = (1 << 26) + 3
    q = torch.zeros(rows, 1, 64, dtype=torch.float16, device="cuda")
    q[-12:] = torch.randn(12, 1, 64, generator=torch.Generator().manual_seed(2)).half().cuda()
    last = q[-12:].clone()
    positions = torch.arange(rows, dtype=torch.int32, device="cuda")
    inv_freq = torch.tensor(W.wq_rope_frequencies(64, 10000.0)[0]).cuda()
    ctx = W.Context(0)
    want = W.wq_rope(ctx, last, None, positions[-12:], inv_freq)[0]
    W.wq_rope(ctx, q, None, positions, inv_freq, q_out=q)
    assert torch.equal(q[-12:], want) and not bool(q[:1000].any()) and not bool(q[-1012:-12].any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout,rot", [(W.ROPE_HALF, 64), (W.ROPE_PAIRS, 64), (W.ROPE_HALF, 16)])
def test_append_is_rope_then_append(dtype, layout, rot):
    B, Hq, Hkv, hd = 5, 14, 2, 64
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    q, k, v = _inputs(B, Hq, Hkv, hd, dtype, 3)
    positions = R.i32([0, 17, 12800, 1 << 20, 5])
    inv_freq = torch.tensor(W.wq_rope_frequencies(rot, 1000000.0)[0]).cuda()
    mk = lambda: R.make_cache(np.random.default_rng(4), [(0, 0, 0, n) for n in (0, 1, 31, 32, 70)], Hkv, hd, 32, t16, slack=2)[0]  # noqa: E731
    one, two = mk(), mk()
    one.len16[4] += 2                       # a full segment
    two.len16[4] += 2
    ctx = W.Context(0)
    for step in range(2):
        qo = W.wq_rope_append_kv(ctx, q, k, v, positions + step, inv_freq, one, layout, 1.25)
        q2, k2 = W.wq_rope(ctx, q, k, positions + step, inv_freq, layout, 1.25)
        assert ctx.device_status() == W.DEV_SEG16_OVERFLOW
        W.wq_append_kv(ctx, k2, v.contiguous(), two)
        assert ctx.device_status() == W.DEV_SEG16_OVERFLOW
        assert torch.equal(qo, q2)
        assert torch.equal(one.len16, two.len16)
        assert torch.equal(one.k16.view(torch.int16), two.k16.view(torch.int16)) and torch.equal(one.v16.view(torch.int16), two.v16.view(torch.int16))
    assert one.len16.tolist() == [2, 3, 33, 34, 72]


def test_captured_steps_append_one_row_each():
    B, Hq, Hkv, hd = 3, 28, 4, 128
    q, k, v = _inputs(B, Hq, Hkv, hd, torch.bfloat16, 9)
    positions = R.i32([4, 5, 6])
    inv_freq = torch.tensor(W.wq_rope_frequencies(hd, 10000.0)[0]).cuda()
    kv = R.make_cache(np.random.default_rng(1), [(0, 0, 0, 4)] * B, Hkv, hd, 64, torch.bfloat16, slack=12)[0]
    stream = torch.cuda.Stream()
    ctx = W.Context(0, stream=stream)
    out = torch.empty(B, Hq, hd, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        W.wq_rope_append_kv(ctx, q, k, v, positions, inv_freq, kv, q_out=out)
        positions.add_(1)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = R.rope(k.double().cpu(), torch.tensor([4, 5, 6]) + step, inv_freq.cpu(), W.ROPE_HALF, 1.0)[0]
        row = kv.k16.view(B, 16, Hkv, hd)[:, 4 + step].double().cpu()
        assert float((row - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) and kv.len16.tolist() == [5 + step] * B
        assert torch.equal(kv.v16.view(B, 16, Hkv, hd)[:, 4 + step], v)
