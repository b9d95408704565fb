"""Attention of a prompt's rows against plain attention in 64 bits: lengths, masks, strides, splits, rows that see nothing."""
import math

import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _case(new, rows, Hq, Hkv, hd, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    channel = torch.exp(torch.randn(Hkv, hd, generator=g))
    fit = (2 * math.sqrt(hd) / channel.norm(dim=-1)).repeat_interleave(Hq // Hkv)[:, None]
    # queries, keys and values cut out of wider rows
    k = (torch.randn(sum(rows) + 1, Hkv, hd, generator=g) * channel * spread).to(dtype).cuda()
    v = (torch.randn(sum(rows) + 1, Hkv, hd, generator=g) * spread).to(dtype).cuda()
    kv = torch.cat([k.flatten(1), v.flatten(1)], 1)
    kv[-1] = math.nan                                    # the row behind the last sequence
    q = (torch.randn(sum(new) + 2, Hq, hd, generator=g) * fit / spread).to(dtype).cuda()
    n = Hkv * hd
    return q, kv[:, :n].unflatten(-1, (Hkv, hd)), kv[:, n:].unflatten(-1, (Hkv, hd))


def _check(new, rows, prefix, Hq, Hkv, hd, dtype, splits, seed=1, spread=1.0, every=1):
    """Compares every `every`-th row of a sequence, and its last."""
    q, k, v = _case(new, rows, Hq, Hkv, hd, dtype, seed, spread)
    q_off, kv_off = R.offsets(new), R.offsets(rows)
    scale = 1.0 / math.sqrt(hd)
    ctx = W.Context(W.prefill_workspace_bytes(q.shape[0], len(new), Hq, Hkv, hd, max(rows), splits))
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    args = (R.i32(q_off), R.i32(kv_off), scale, None if prefix is None else R.i32(prefix), max(rows), splits)
    W.wq_prefill_attention(ctx, q, k, v, *args, out=out, lse=lse)
    again = W.wq_prefill_attention(ctx, q, k, v, *args, out=torch.full_like(q, 7.0))
    assert torch.equal(again, out), "two calls differ"
    assert bool((out[q_off[-1]:] == 7.0).all()) and bool((lse[q_off[-1]:] == 7.0).all()), "rows behind the last sequence"
    u = R.HALF_STEP[dtype]
    for b, n in enumerate(new):
        if n == 0:
            continue
        L = rows[b]
        p = 0 if prefix is None else min(max(prefix[b], 0), L)
        picked = list(range(0, n, every)) + ([n - 1] if (n - 1) % every else [])
        limit = [max(L - n + i + 1, p) for i in picked]
        qs, ks = [q_off[b] + i for i in picked], slice(kv_off[b], kv_off[b + 1])
        want, want_lse, spread_v, terms = R.attend(q[qs].double().cpu(), k[ks].double().cpu(), v[ks].double().cpu(), limit, scale)
        got, got_lse = out[qs].double().cpu(), lse[qs].double().cpu()
        seen = torch.isfinite(want_lse)
        assert torch.equal(seen, torch.isfinite(got_lse)) and bool((got[~seen] == 0).all()) and bool((got_lse[~seen] == -math.inf).all())
        if not seen.any():
            continue
        w = R.weights_error(L, hd, terms, float(want_lse[seen].abs().max()))
        # weights rounded to the type (none in fp32), their errors, the result's rounding; a fp16 weight below 2^-34 of the largest is off by
        # up to half of fp16's smallest step, 2^-35 of the largest weight
        bound = ((0.0 if dtype == torch.float32 else u) + 2 * w) * spread_v + u * want.abs()
        if dtype == torch.float16:
            bound = bound + 2.0 ** -35 * v[ks].double().cpu().abs().sum(0).repeat_interleave(Hq // Hkv, 0) + 2.0 ** -25
        assert bool(((got - want).abs()[seen] <= bound[seen]).all()), (b, float(((got - want).abs() / bound)[seen].max()))
        assert bool(((got_lse - want_lse).abs()[seen] <= 2 * w + 2.0 ** -22 * want_lse.abs()[seen]).all())


SMALL, LARGE = (14, 2, 64), (28, 4, 128)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [SMALL, LARGE, (8, 8, 64), (3, 3, 128), (16, 2, 128)])
def test_ragged_batches(dtype, heads):
    rows = [1, 64, 65, 200, 18, 0, 127, 3]
    _check(rows, rows, None, *heads, dtype, 1)
    _check(rows, rows, [0, 64, 30, 150, 99, 5, -3, 2], *heads, dtype, 0, seed=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("splits", [0, 1, 3, 64])
def test_chunks_and_single_tokens(dtype, splits):
    _check([1, 1, 1, 1], [1, 130, 777, 64], None, *SMALL, dtype, splits)
    _check([5, 61, 1], [700, 1000, 333], [0, 990, 100], *LARGE, dtype, splits)


@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("heads", [SMALL, LARGE, (16, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("splits", [0, 1, 5, 64])
def test_few_rows_each(dtype, heads, splits):
    """At most 16 products' columns a sequence on the average; some have more, none, or fewer keys than queries."""
    _check([1, 1, 0, 8, 1, 1], [31, 33, 40, 600, 2100, 1], None, *heads, dtype, splits, seed=3)
    _check([1, 4, 1, 1, 0, 2], [256, 2, 0, 257, 0, 512], [0, 2, 0, 256, 0, 511], *heads, dtype, splits, seed=4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("splits", [1, 4])
def test_rows_that_see_nothing(dtype, splits):
    # more queries than keys: the first ones have positions in front of the first key; no keys at all
    _check([70, 9, 20], [40, 0, 19], None, *SMALL, dtype, splits)
    _check([70, 9, 20], [40, 0, 19], [1, 4, 0], *SMALL, dtype, splits)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread", [2.0 ** -10, 2.0 ** 6])
def test_magnitudes(dtype, spread):
    _check([150], [150], [100], *SMALL, dtype, 1, spread=spread)


def test_long_rows():
    _check([700], [2500], [1000], 4, 2, 128, torch.bfloat16, 0)
    _check([2300], [2300], [2000], 2, 1, 64, torch.float16, 1)


@pytest.mark.parametrize("dtype", DTYPES[:2])
def test_a_last_round_of_tiles(dtype):
    """More tiles than compute units: the last ones are cut along the keys.  One sequence and two, with tiles that see little or nothing."""
    _check([4400], [4400], [4400], 16, 16, 64, dtype, 0, every=37)
    _check([1300], [2500], [2000], 56, 8, 128, dtype, 0, every=11)
    _check([1300], [1000], [0], 56, 8, 128, dtype, 0, every=11)
    _check([2800], [2800], [2800], 24, 3, 64, dtype, 0, every=53)       # (a last round that ends inside a tile's KV heads)
    _check([300, 4200], [300, 4200], [10, 3000], 16, 16, 64, dtype, 0, every=37)


@pytest.mark.parametrize("new", [[300], [3], [40]])
def test_rows_far_apart(new):
    """Keys and values 2^22 elements from row to row: 5.9 GB, offsets of more than 32 bits."""
    Hq, Hkv, hd, rows = 8, 2, 128, 700
    g = torch.Generator().manual_seed(8)
    wide = torch.empty(rows, 1 << 22, dtype=torch.float16, device="cuda")
    n = Hkv * hd
    wide[:, :n] = torch.randn(rows, n, generator=g).half().cuda()
    wide[:, -n:] = torch.randn(rows, n, generator=g).half().cuda()
    k, v = wide[:, :n].unflatten(-1, (Hkv, hd)), wide[:, -n:].unflatten(-1, (Hkv, hd))
    q = torch.randn(sum(new), Hq, hd, generator=g).half().cuda()
    ctx = W.Context(W.prefill_workspace_bytes(sum(new), 1, Hq, Hkv, hd, rows))
    a = [W.wq_prefill_attention(ctx, q, x, y, R.i32(R.offsets(new)), R.i32([0, rows]), 0.09, None, rows) for x, y in ((k, v), (k.contiguous(), v.contiguous()))]
    assert torch.equal(a[0], a[1]) and bool(a[0].isfinite().all())


def test_steep_and_rising_logits():
    """Every key's logit above the one before (the reference moves again and again), and one key that takes all weight."""
    hd, L = 64, 400
    for dtype in DTYPES:
        for logits in (torch.linspace(-150, 150, L), torch.linspace(150, -150, L), torch.where(torch.arange(L) == 77, 200.0, 0.0)):
            k = torch.zeros(L, 1, hd, dtype=dtype)
            k[:, 0, 0] = logits.to(dtype)
            v = torch.randn(L, 1, hd, generator=torch.Generator().manual_seed(0)).to(dtype)
            q = torch.zeros(1, 1, hd, dtype=dtype)
            q[..., 0] = 1.0
            ctx = W.Context(W.prefill_workspace_bytes(1, 1, 1, 1, hd, L, 4))
            for splits in (1, 4):
                out = W.wq_prefill_attention(ctx, q.cuda(), k.cuda(), v.cuda(), R.i32([0, 1]), R.i32([0, L]), 1.0, num_splits=splits)
                want, _, spread, terms = R.attend(q.double(), k.double(), v.double(), [L], 1.0)
                bound = (R.HALF_STEP[dtype] * 2 + 2 * R.weights_error(L, hd, terms, 200)) * spread + 2.0 ** -25
                assert bool(((out.double().cpu() - want).abs() <= bound).all())


def test_a_stream_of_its_own_and_a_graph():
    new, heads = [33, 1, 90], LARGE
    q, k, v = _case(new, [50, 300, 90], *heads, torch.bfloat16, 5)
    q_off, kv_off = R.i32(R.offsets(new)), R.i32(R.offsets([50, 300, 90]))
    need = W.prefill_workspace_bytes(q.shape[0], 3, *heads, 300, 3)
    want = W.wq_prefill_attention(W.Context(need), q, k, v, q_off, kv_off, 0.1, num_splits=3, out=torch.zeros_like(q))
    stream = torch.cuda.Stream()
    ctx = W.Context(need, stream=stream)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        W.wq_prefill_attention(ctx, q, k, v, q_off, kv_off, 0.1, num_splits=3, out=out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
