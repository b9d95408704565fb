"""Attention of several new rows per sequence over its packed cache and each other, against plain attention in 64 bits over the same values."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import tree_ref as T

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
SMALL, LARGE = (14, 2, 64), (28, 4, 128)


def _inputs(rng, rows, heads, dtype, scale=1.0, spread_q=1.0, fused=True):
    Hq, Hkv, hd = heads
    x = rng.normal(0, 1, (rows, Hq + 2 * Hkv, hd))
    x[:, :Hq] *= 2.0 / (scale * 1.5) * spread_q
    x[:, Hq:] *= scale
    x = torch.from_numpy(x).to(dtype).cuda()
    parts = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return parts if fused else tuple(p.contiguous() for p in parts)


def _compare(got, got_lse, q, k, v, sees, sm, dtype):
    """One sequence's rows; returns the squares of the errors and of the values."""
    want, want_lse, spread, terms = T.attend(q.double().cpu(), k, v, sees, sm)
    u, exact = R.HALF_STEP[dtype], dtype == torch.float32
    w = R.weights_error(k.shape[0], q.shape[-1], terms, float(want_lse.abs().max()))
    # 16-bit types: packed keys rounded to 11 bits (of every product of a logit), weights to the type that meets the values, packed values to 11 bits;
    # the result once.  A logit's error moves every weight, and their sum
    soft = 0.0 if exact else 2.0 ** -11 * terms + u + 2 * 2.0 ** -11
    bound = (2 * w + soft) * spread + u * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    if not exact:
        # (weights below 2^-24 of fp16's range, 2^-35 of the largest, are lost)
        bound = bound + 2.0 ** -11 * terms * want.abs() + 2.0 ** -35 * v.abs().sum(0).repeat_interleave(q.shape[1] // v.shape[1], 0)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    assert bool(((got_lse.double().cpu() - want_lse).abs() <= 2 * w + 2.0 ** -22 * want_lse.abs() + (0.0 if exact else 2.0 ** -11 * terms)).all())
    return float(err.square().sum()), float(want.square().sum())


def _check(lens, rows, heads, group, dtype, parents="random", splits=0, front=0, behind=0, seed=1, scale=1.0, spread_q=1.0, hints=True, fused=True):
    """lens[b] = tokens per class, rows[b] = new rows; parents: None (chains), "random", or one list a sequence.  `front` and `behind` rows belong to nobody."""
    Hq, Hkv, hd = heads
    rng = np.random.default_rng(seed)
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    kv, cached = R.make_cache(rng, lens, Hkv, hd, group, t16, slack=2, scale=scale)
    off = [front + x for x in R.offsets(rows)]
    total = off[-1] + behind
    if parents == "random":
        parents = [T.random_tree(rng, n, 1 + b % 2) for b, n in enumerate(rows)]
    q, k, v = _inputs(rng, total, heads, dtype, scale, spread_q, fused)
    sm = 1.0 / math.sqrt(hd)
    longest, most = (max(sum(x) for x in lens), max(rows)) if hints else (0, 0)
    ctx = W.Context(W.tree_workspace_bytes(total, len(lens), Hq, Hkv, hd, longest, most, splits))
    parent = None if parents is None else R.i32([-1] * front + sum(parents, []) + [-1] * behind)
    out = torch.full((total, Hq, hd), 77.0, dtype=dtype, device="cuda")
    lse = torch.full((total, Hq), 77.0, device="cuda")
    assert W.wq_tree_attention(ctx, q, k, v, kv, R.i32(off), sm, parent, most, longest, splits, out, lse) is out
    alone = torch.full_like(out, 77.0)                       # without lse: other kernels for bf16
    W.wq_tree_attention(ctx, q, k, v, kv, R.i32(off), sm, parent, most, longest, splits, alone)
    assert ctx.device_status() == 0
    for x in (out, lse, alone):
        assert bool((x[:front] == 77).all()) and bool((x[off[-1]:] == 77).all())
    num = den = 0.0
    for b, n in enumerate(rows):
        if n == 0:
            continue
        s = slice(off[b], off[b + 1])
        kk, vv = (torch.cat([c, x[s].double().cpu()]) for c, x in zip(cached[b], (k, v)))
        sees = torch.cat([torch.ones(n, cached[b][0].shape[0], dtype=torch.bool), T.seen(None if parents is None else parents[b], n)], 1)
        for got in (out, alone):
            e, d = _compare(got[s], lse[s], q[s], kk, vv, sees, sm, dtype)
            num, den = num + e, den + d
    # roundings are independent: their common size is well below the worst case.  Output and weights at u (rms u / sqrt 3 each), values at 2^-11, a
    # logit of deviation 2 by 2^-11 of its terms
    if dtype != torch.float32 and spread_q == 1.0:
        assert math.sqrt(num / den) <= 1.5 * R.HALF_STEP[dtype] + 6 * 2.0 ** -11, math.sqrt(num / den)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (SMALL, 64), (LARGE, 64), (LARGE, 32), (LARGE, 128), ((8, 8, 64), 32), ((16, 2, 128), 64), ((3, 3, 128), 32)])
def test_trees_over_mixed_caches(dtype, heads, group):
    _check([(100, 64, 33, 20), (0, 40, 0, 3), (7, 0, 90, 0)], [5, 1, 19], heads, group, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (LARGE, 64), ((8, 8, 64), 64)])
def test_chains(dtype, heads, group):
    _check([(100, 64, 33, 20), (0, 40, 0, 3), (0, 0, 0, 0), (0, 0, 0, 9)], [9, 1, 70, 0], heads, group, dtype, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [(1, 0, 0, 0), (0, 31, 0, 0), (0, 0, 65, 0), (0, 0, 0, 1), (0, 0, 0, 200), (33, 0, 0, 64), (0, 0, 0, 0)])
@pytest.mark.parametrize("splits", [1, 5])
def test_single_classes_and_tiny_caches(dtype, lens, splits):
    for parents in (None, "random"):
        _check([lens], [1], SMALL, 32, dtype, parents, splits)
        _check([lens], [6], LARGE, 64, dtype, parents, splits)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_nobody_and_sequences_without_rows(dtype):
    _check([(32, 0, 7, 3), (0, 0, 0, 0), (70, 130, 10, 0), (5, 5, 5, 5)], [0, 4, 0, 21], SMALL, 32, dtype, front=3, behind=2)
    _check([(32, 0, 7, 3), (0, 0, 0, 0), (70, 130, 10, 0), (5, 5, 5, 5)], [3, 0, 2, 0], LARGE, 64, dtype, None, front=1, behind=70, splits=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [SMALL, (3, 3, 64), (4, 2, 128)])
def test_more_rows_than_a_workgroup_takes(dtype, heads):
    _check([(64, 96, 0, 11), (0, 0, 32, 0)], [300, 41], heads, 32, dtype)
    _check([(64, 96, 0, 11), (0, 0, 32, 0)], [300, 41], heads, 64, dtype, None, 3, fused=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [63, 64, 65, 128, 200])
def test_ends_of_tiles(dtype, n):
    _check([(0, n, 0, 130 - n % 64)], [n], (4, 2, 64), 32, dtype)
    _check([(0, n, 0, 130 - n % 64)], [n], (4, 2, 64), 32, dtype, None, splits=4)


@pytest.mark.parametrize("shape", ["line", "star", "comb", "random"])
def test_largest_trees(shape):
    n = 1024
    rng = np.random.default_rng(3)
    parent = {"line": [i - 1 for i in range(n)], "star": [-1] + [0] * (n - 1), "comb": [i - 1 if i % 2 == 0 else max(i - 2, 0) if i > 1 else 0 for i in range(n)],
              "random": T.random_tree(rng, n)}[shape]
    parent[0] = -1
    _check([(32, 0, 0, 40)], [n], (2, 2, 64), 64, torch.bfloat16, [parent])
    _check([(32, 0, 0, 40), (0, 9, 0, 0)], [n, 3], (7, 1, 64), 32, torch.float32, [parent, [-1, 0, 0]], splits=2)


def test_values_that_are_no_parents():
    bad = [[0, 1, 2, -5, 99, 1 << 30, 3, -(1 << 31), 7], [5, 0, 1, 3]]
    for dtype in DTYPES:
        _check([(0, 33, 0, 4), (9, 0, 0, 0)], [9, 4], SMALL, 32, dtype, bad)


def test_a_tree_with_too_many_rows():
    Hq, Hkv, hd, n = 4, 2, 64, 1100
    rng = np.random.default_rng(8)
    kv, cached = R.make_cache(rng, [(0, 40, 0, 3), (0, 0, 9, 0)], Hkv, hd, 32, torch.bfloat16)
    q, k, v = _inputs(rng, n + 2, (Hq, Hkv, hd), torch.bfloat16)
    parents = [T.random_tree(rng, n), [-1, 0]]
    for splits in (1, 4):
        ctx = W.Context(W.tree_workspace_bytes(n + 2, 2, Hq, Hkv, hd, 50, 1024, splits))
        lse = torch.full((n + 2, Hq), 77.0, device="cuda")
        out = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, n, n + 2]), 0.125, R.i32(sum(parents, [])), 1024, 50, splits, lse=lse)
        assert ctx.device_status() == W.DEV_TOO_MANY_ROWS
        assert bool((out[1024:n] == 0).all()) and bool((lse[1024:n] == -math.inf).all())
        for b, s in ((0, slice(0, 1024)), (1, slice(n, n + 2))):
            kk, vv = (torch.cat([c, x[s].double().cpu()]) for c, x in zip(cached[b], (k, v)))
            rows = s.stop - s.start
            sees = torch.cat([torch.ones(rows, cached[b][0].shape[0], dtype=torch.bool), T.seen(parents[b][:rows], rows)], 1)
            _compare(out[s], lse[s], q[s], kk, vv, sees, 0.125, torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,most,chain", [([40, 3, 9], 5, True), ([300, 0, 70], 20, True), ([60, 4, 0], 8, False), ([5, 6, 5], 5, False), ([700, 650, 3], 640, True)])
def test_sequences_with_more_rows_than_the_caller_said(dtype, rows, most, chain):
    Hq, Hkv, hd = 14, 2, 64
    rng = np.random.default_rng(9)
    kv, cached = R.make_cache(rng, [(0, 40, 0, 3), (0, 0, 9, 0), (64, 0, 1, 33)], Hkv, hd, 32, torch.bfloat16 if dtype == torch.bfloat16 else torch.float16)
    off = np.cumsum([0] + rows)
    total = int(off[-1])
    q, k, v = _inputs(rng, total + 2, (Hq, Hkv, hd), dtype)          # (the last two rows belong to nobody)
    parents = [T.random_tree(rng, n) for n in rows]
    for splits in (0, 1, 3):
        ctx = W.Context(max(1 << 22, W.tree_workspace_bytes(total + 2, 3, Hq, Hkv, hd, 98, most, splits)))
        out, lse = torch.full((total + 2, Hq, hd), 77.0, device="cuda", dtype=dtype), torch.full((total + 2, Hq), 77.0, device="cuda")
        parent = None if chain else R.i32(sum(parents, []) + [0, 0])
        W.wq_tree_attention(ctx, q, k, v, kv, R.i32(off), 0.125, parent, most, 98, splits, out, lse)
        assert ctx.device_status() == W.DEV_TOO_MANY_ROWS
        assert bool((out[total:] == 77).all()) and bool((lse[total:] == 77).all())
        for b, n in enumerate(rows):
            a, m = int(off[b]), min(n, most)
            assert bool((out[a + m:a + n] == 0).all()) and bool((lse[a + m:a + n] == -math.inf).all())
            if not m:
                continue
            s = slice(a, a + m)
            kk, vv = (torch.cat([c, x[s].double().cpu()]) for c, x in zip(cached[b], (k, v)))
            new = torch.tril(torch.ones(m, m, dtype=torch.bool)) if chain else T.seen(parents[b][:m], m)
            _compare(out[s], lse[s], q[s], kk, vv, torch.cat([torch.ones(m, cached[b][0].shape[0], dtype=torch.bool), new], 1), 0.125, dtype)


def test_long_caches():
    _check([(2500, 2000, 1100, 150)], [40], (14, 2, 128), 64, torch.bfloat16)
    _check([(2500, 2000, 1100, 150), (9, 0, 0, 4000)], [4, 2], LARGE, 64, torch.bfloat16)
    _check([(700, 0, 1100, 1250)], [3], SMALL, 64, torch.float16, None)
    _check([(700, 900, 300, 50)], [2], LARGE, 32, torch.float32)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 9, 10, 16, 18, 19, 30, 33, 36, 37])
def test_numbers_of_rows(rows):
    """From one row to more than any kernel's columns, over enough keys for several parts."""
    for heads, group in ((LARGE, 64), (SMALL, 32), ((8, 8, 128), 128)):
        _check([(700, 330, 90, 70), (0, 65, 0, 900)], [rows, max(1, rows - 2)], heads, group, torch.bfloat16, "random" if rows % 2 else None)
    _check([(700, 330, 90, 70)], [rows], LARGE, 32, torch.float16)


def test_bounds_that_are_not_given():
    for dtype in DTYPES:
        _check([(100, 64, 33, 20), (0, 40, 0, 3)], [5, 40], LARGE, 64, dtype, hints=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale,spread_q", [(2.0 ** -6, 1.0), (2.0 ** 5, 1.0), (1.0, 2.0 ** 4)])
def test_magnitudes(dtype, scale, spread_q):
    if spread_q == 1.0 or dtype == torch.float32:
        _check([(64, 96, 40, 30)], [7], LARGE if spread_q == 1.0 else SMALL, 32, dtype, scale=scale, spread_q=spread_q)


@pytest.mark.parametrize("dtype", DTYPES)
def test_queries_that_are_not_finite(dtype):
    """A row with NaN or infinity in its query becomes NaN; the others keep their results bit for bit."""
    rng = np.random.default_rng(2)
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    for lens in ((64, 40, 33, 20), (0, 0, 0, 0), (0, 0, 0, 50)):
        kv, _ = R.make_cache(rng, [lens], 4, 128, 64, t16)
        q, k, v = _inputs(rng, 6, LARGE, dtype, fused=False)
        parent = R.i32([-1, 0, 0, 1, 1, 2])
        ctx = W.Context(W.tree_workspace_bytes(6, 1, 28, 4, 128, 200, 6))
        lse, lse2 = (torch.empty(6, 28, device="cuda") for _ in range(2))
        clean = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, 6]), 0.1, parent, 6, 200, lse=lse).clone()
        q[2, 5, 9] = math.nan
        dirty = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, 6]), 0.1, parent, 6, 200, lse=lse2)
        bad = torch.zeros(6, 28, dtype=torch.bool, device="cuda")
        bad[2, 5] = True
        assert bool(dirty[bad].isnan().all()) and bool(lse2[bad].isnan().all())
        assert torch.equal(dirty[~bad], clean[~bad]) and torch.equal(lse2[~bad], lse[~bad])


def test_hidden_keys_that_are_not_finite():
    """NaN and infinity in the key of a row that others do not see change nothing for them but roundings (a wavefront's rows move the references of their
    exponents together)."""
    rng = np.random.default_rng(2)
    for dtype in DTYPES:
        t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
        kv, cached = R.make_cache(rng, [(0, 40, 0, 20)], 2, 64, 32, t16)
        q, k, v = _inputs(rng, 6, SMALL, dtype, fused=False)
        parents = [-1, 0, 0, 1, 1, 2]
        ctx = W.Context(W.tree_workspace_bytes(6, 1, 14, 2, 64, 60, 6))
        kk, vv = (torch.cat([c, x.double().cpu()]) for c, x in zip(cached[0], (k, v)))
        k[3, 1, 7], k[5, 0, 0], k[5, 1, 0] = math.nan, math.inf, -math.inf
        lse = torch.empty(6, 14, device="cuda")
        out = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, 6]), 0.1, R.i32(parents), 6, 60, lse=lse)
        sees = torch.cat([torch.ones(6, 60, dtype=torch.bool), T.seen(parents, 6)], 1)
        rows = [0, 1, 2, 4]
        _compare(out[rows], lse[rows], q[rows], kk, vv, sees[rows], 0.1, dtype)
        assert bool(out[3, 7:].isnan().all()) and bool(lse[3, 7:].isnan().all())


def test_bf16_queries_beyond_fp16():
    rng = np.random.default_rng(0)
    kv, _ = R.make_cache(rng, [(50, 40, 30, 20)], 4, 128, 64, torch.bfloat16)
    q, k, v = _inputs(rng, 5, LARGE, torch.bfloat16)
    ctx = W.Context(W.tree_workspace_bytes(5, 1, 28, 4, 128, 140, 5))
    for e in (-60, 60):
        big = (q.double() * 2.0 ** e).to(torch.bfloat16)
        a = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, 5]), 0.125, None, 5, 140)
        b = W.wq_tree_attention(ctx, big, k, v, kv, R.i32([0, 5]), 0.125 * 2.0 ** -e, None, 5, 140)
        assert torch.equal(a, b)


def test_one_row_is_a_decode_step():
    """One new row per sequence: what wq_decode_append_attention gives, within that kernel's 2e-3 of a vector's largest entry and a rounding."""
    rng = np.random.default_rng(4)
    lens = [(640, 330, 90, 70), (0, 65, 0, 9), (32, 0, 0, 0)]
    kv, _ = R.make_cache(rng, lens, 4, 128, 64, torch.bfloat16, slack=1)
    q, k, v = _inputs(rng, 3, LARGE, torch.bfloat16, fused=False)
    ctx = W.Context(max(W.tree_workspace_bytes(3, 3, 28, 4, 128, 1200, 1), W.workspace_bytes(3, 28, 128, 8)))
    a = W.wq_tree_attention(ctx, q, k, v, kv, R.i32([0, 1, 2, 3]), 0.088, None, 1, 1200).double()
    b = W.wq_decode_append_attention(ctx, q, kv, k, v, 0.088, 4).double()
    assert bool(((a - b).abs() <= 2e-3 * b.abs().amax(-1, keepdim=True) + 2.0 ** -8 * b.abs() + 4e-3 * b.abs().amax(-1, keepdim=True)).all())


def test_fewer_parts_where_the_workspace_is_small():
    rng = np.random.default_rng(6)
    kv, _ = R.make_cache(rng, [(1500, 700, 300, 60)], 2, 64, 32, torch.float16)
    q, k, v = _inputs(rng, 4, SMALL, torch.float32)
    full = W.tree_workspace_bytes(4, 1, 14, 2, 64, 2560, 4)
    outs = []
    for ws in (full, 16384 + 4 * 14 * 66 * 4 * 3, 16384):
        outs.append(W.wq_tree_attention(W.Context(ws), q, k, v, kv, R.i32([0, 4]), 0.125, None, 4, 2560))
    for x in outs[1:]:
        assert float((x - outs[0]).abs().max()) <= 2e-5 * float(outs[0].abs().max())


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_segment_far_into_its_buffers(dtype):
    """8-bit codes and 16-bit rows of which the last ones are used: 5.2 GB of codes, 4.3 GB of rows; new rows 2^22 elements apart."""
    hd, t16 = 64, torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    near, _ = R.make_cache(np.random.default_rng(5), [(0, 0, 190, 77)], 2, hd, 32, t16)
    far16, far = 1 << 24, 20480000
    wide = W.PackedKV(1, 2, hd, 32, t16, [0, 0, far + near.cap[2]], [far16, far16 + 77])
    wide.codes[2][:, :, far * hd:] = near.codes[2]
    wide.meta[2][:, :, far * 2:] = near.meta[2]
    wide.cls_off[2].copy_(near.cls_off[2] + far)
    wide.cls_len[2].copy_(near.cls_len[2])
    wide.k16[far16:], wide.v16[far16:] = near.k16, near.v16
    wide.len16.copy_(near.len16)
    g = torch.Generator().manual_seed(1)
    n, apart = (600 if dtype != torch.float32 else 300), 1 << 22
    room = torch.empty((n - 1) * apart + 4096, dtype=dtype, device="cuda")
    k = room[:(n - 1) * apart + 128].as_strided((n, 2, hd), (apart, hd, 1))
    v = room[1024:].as_strided((n, 2, hd), (apart, hd, 1))
    x = torch.randn(2, n, 2, hd, generator=g).to(dtype).cuda()
    k.copy_(x[0])
    v.copy_(x[1])
    q = torch.randn(n, 4, hd, generator=g).to(dtype).cuda()
    ctx = W.Context(W.tree_workspace_bytes(n, 1, 4, 2, hd, 300, n))
    a = W.wq_tree_attention(ctx, q, x[0], x[1], near, R.i32([0, n]), 0.1, None, n, 300)
    b = W.wq_tree_attention(ctx, q, k, v, wide, R.i32([0, n]), 0.1, None, n, 300)
    assert torch.equal(a, b) and bool(a.isfinite().all())


def test_on_a_stream_in_a_graph():
    """Captured once, replayed over a cache that grows and other rows in between, with eager work between the replays; two graphs share the workspace."""
    rng = np.random.default_rng(9)
    kv, cached = R.make_cache(rng, [(200, 64, 33, 20), (0, 90, 0, 3)], 4, 128, 64, torch.bfloat16, slack=8)
    q, k, v = _inputs(rng, 12, LARGE, torch.bfloat16, fused=False)
    off, parent = R.i32([0, 7, 12]), R.i32(T.random_tree(rng, 7) + T.random_tree(rng, 5))
    stream = torch.cuda.Stream()
    ctx = W.Context(W.tree_workspace_bytes(12, 2, 28, 4, 128, 400, 7), stream=stream)
    torch.cuda.synchronize()
    outs, graphs = [], []
    with torch.cuda.stream(stream):
        for chain in (False, True):
            out, graph = torch.zeros(12, 28, 128, dtype=torch.bfloat16, device="cuda"), torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                W.wq_tree_attention(ctx, q, k, v, kv, off, 0.0884, None if chain else parent, 7, 400, out=out)
            outs.append(out)
            graphs.append(graph)
        for step in range(4):
            for graph in graphs:
                graph.replay()
            got = [x.clone() for x in outs]
            for chain in (False, True):
                want = W.wq_tree_attention(ctx, q, k, v, kv, off, 0.0884, None if chain else parent, 7, 400)
                assert torch.equal(got[chain], want), (step, chain)
            W.wq_append_kv(ctx, k[step:step + 2].contiguous(), v[step:step + 2].contiguous(), kv)
            q.mul_(-1)
            torch.cuda.synchronize()
        assert ctx.device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_sequences(dtype):
    rng = np.random.default_rng(11)
    lens = [(int(rng.integers(0, 40)), int(rng.integers(0, 70)), 0, int(rng.integers(0, 9))) for _ in range(150)]
    _check(lens, [int(x) for x in rng.integers(0, 4, 150)], (7, 1, 64), 32, dtype)
    _check(lens, [int(x) for x in rng.integers(0, 30, 150)], (7, 1, 64), 32, dtype, None, hints=False)


def test_calls_on_two_streams_at_once():
    """A context and a workspace each; what both give is what one after the other gives."""
    rng = np.random.default_rng(12)
    kv, _ = R.make_cache(rng, [(900, 700, 300, 60), (64, 0, 33, 5)], 4, 128, 64, torch.bfloat16)
    sets = []
    for n in (6, 40):
        q, k, v = _inputs(rng, 2 * n, (28, 4, 128), torch.bfloat16)
        ctx = W.Context(W.tree_workspace_bytes(2 * n, 2, 28, 4, 128, 2000, n))
        sets.append((ctx, q, k, v, R.i32([0, n, 2 * n]), R.i32(T.random_tree(rng, n) + T.random_tree(rng, n)), n, torch.cuda.Stream()))
    call = lambda s, out=None: W.wq_tree_attention(s[0], s[1], s[2], s[3], kv, s[4], 0.0884, s[5], s[6], 2000, out=out)      # noqa: E731
    want = [call(s) for s in sets]
    torch.cuda.synchronize()
    outs = [torch.empty_like(w) for w in want]
    for s in sets:
        s[0].set_stream(s[-1])
    for _ in range(10):
        for s, out in zip(sets, outs):
            call(s, out)
    torch.cuda.synchronize()
    for out, w, s in zip(outs, want, sets):
        assert torch.equal(out, w) and s[0].device_status() == 0
