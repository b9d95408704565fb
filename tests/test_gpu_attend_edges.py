"""Prompt attention and shared decode where a call is out of the ordinary: a workspace that was sized for another call, queries of zero and scales at the
ends of fp32, NaN, values far beyond fp16, and how much of a 16-bit call's accuracy its roundings take."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import test_gpu_prefill as P
from tests import test_gpu_shared_prefix as S

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
SMALL, LARGE = (14, 2, 64), (28, 4, 128)


# ---- a workspace that was sized for another call ---------------------------------------------------------------------
@pytest.mark.parametrize("new,rows,prefix,heads,largest", [
    ([400], [6400], [0], LARGE, (6400, 6400)),                     # parts, where the largest call has none
    ([1, 1, 1], [900, 6400, 77], None, SMALL, (8000, 6400)),       # ... of single tokens
    ([4400], [4400], [4400], (16, 16, 64), (6400, 6400)),          # a cut last round, where the largest call has none
    ([4400], [4400], [4400], (16, 16, 64), None),                  # room for some of its parts
    ([40], [3000], None, LARGE, None)])
def test_prompts_on_a_workspace_for_a_larger_call(monkeypatch, new, rows, prefix, heads, largest):
    ample = W.prefill_workspace_bytes(sum(new), len(new), *heads, max(rows))
    size = W.prefill_workspace_bytes(largest[0], 1, *heads, largest[1]) if largest else 16384 + (ample - 16384) // 2
    assert 16384 <= size < ample
    monkeypatch.setattr(W, "prefill_workspace_bytes", lambda *a: size)
    P._check(new, rows, prefix, *heads, torch.bfloat16, 0, every=37 if sum(new) > 1000 else 7)


@pytest.mark.parametrize("B,largest,own", [(32, 37, None), (32, 37, (0, 0, 0, 9)), (31, 39, (40, 0, 9, 11)), (30, 37, (0, 0, 0, 1500))])
@pytest.mark.parametrize("dtype", DTYPES[1:])
def test_shared_caches_on_a_workspace_for_a_larger_call(monkeypatch, B, largest, own, dtype):
    longest, longest_own = (2100, sum(own) if own else 0)
    size = W.shared_workspace_bytes(largest, 1, *SMALL, longest, longest_own)
    assert size < W.shared_workspace_bytes(B, 1, *SMALL, longest, longest_own)
    # (and one that holds a single part of everything, the least that any call of this size has been sized for)
    for bytes_ in (size, W.shared_workspace_bytes(B, 1, *SMALL, 1, 1, 1)):
        with monkeypatch.context() as m:
            m.setattr(W, "shared_workspace_bytes", lambda *a: bytes_)
            S._check([(700, 900, 400, 100)], [B], None if own is None else [own] * B, SMALL, 32, dtype)


# ---- queries of zero, scales at the ends of fp32 --------------------------------------------------------------------------------------------------
def _mean_of(kv_logical, heads):
    return kv_logical[1].mean(0).repeat_interleave(heads[0] // heads[1], 0)


@pytest.mark.parametrize("sm", [0.125, 0.125 * 2.0 ** -60, 2.0 ** -149, 2.0 ** 127])
@pytest.mark.parametrize("dtype", DTYPES)
def test_queries_of_zero(dtype, sm):
    """Every key has the same logit, 0, whatever the scale: the mean of the values.  Lengths that end inside a tile."""
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    prefix, logical = R.make_cache(np.random.default_rng(0), [(50, 40, 30, 21)], 2, 64, 32, t16)
    q = torch.zeros(2, 14, 64, dtype=dtype, device="cuda")
    out = W.wq_decode_attention_shared(W.Context(W.shared_workspace_bytes(2, 1, *SMALL, 141)), q, prefix, R.i32([0, 2]), None, sm)
    want = _mean_of(logical[0], SMALL)
    # weights of one are exact; values rounded to fp16, their sum to the type, 141 additions
    size = logical[0][1].abs().mean(0).repeat_interleave(7, 0)
    bound = (0.0 if dtype == torch.float32 else 2.0 ** -11) * size + 160 * 2.0 ** -24 * size + R.HALF_STEP[dtype] * want.abs() + 2.0 ** -25
    assert bool(((out.double().cpu() - want).abs() <= bound).all())
    k, v = prefix.k16[:21], prefix.v16[:21]
    if dtype != torch.float32:
        for n in (1, 19):
            o = W.wq_prefill_attention(W.Context(0), torch.zeros(n, 14, 64, dtype=dtype, device="cuda"), k, v, R.i32([0, n]), R.i32([0, 21]), sm)
            want = torch.stack([v[:21 - n + i + 1].double().mean(0) for i in range(n)]).repeat_interleave(7, 1).cpu()
            assert bool(((o.double().cpu() - want).abs() <= R.HALF_STEP[dtype] * want.abs() + 24 * 2.0 ** -24 * 6 + 2.0 ** -25).all())


def test_large_bf16_queries_over_keys_of_zero():
    """The scale that goes with a bf16 query's power of two is beyond fp32, the logits are 0."""
    kv = W.PackedKV(1, 2, 64, 32, torch.bfloat16, [32, 64, 32], [0, 0], fill=0)
    for c, n in enumerate((20, 64, 7)):
        kv.cls_off[c].copy_(R.i32([0, kv.cap[c]]))
        kv.cls_len[c].fill_(n)
        kv.meta[c][1].fill_(int(np.float16(c + 1.0).view(np.uint16)) << 16)       # values of 1, 2, 3
    q = torch.full((1, 14, 64), 2.0 ** 100, dtype=torch.bfloat16, device="cuda")
    q[0, 3] = 2.0 ** 127
    out = W.wq_decode_attention_shared(W.Context(W.shared_workspace_bytes(1, 1, *SMALL, 91)), q, kv, R.i32([0, 1]), None, 2.0 ** 30)
    want = (20 + 2 * 64 + 3 * 7) / 91
    assert bool(((out.double() - want).abs() <= (2.0 ** -8 + 100 * 2.0 ** -24) * want).all())


# ---- NaN -----------------------------------------------------------------------------------------------------------------
def _nan_where(out, lse, hit):
    assert torch.equal(out.isnan().all(-1), hit) and torch.equal(out.isnan().any(-1), hit), "result"
    assert torch.equal(lse.isnan(), hit) and bool(lse[~hit].isfinite().all()), "log-sum-exp"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,splits", [([90], 1), ([90], 3), ([400], 1), ([2, 1], 1), ([2, 1], 3)])
def test_a_query_that_is_not_a_number(dtype, new, splits):
    """Its own row becomes NaN, and so does that row's log-sum-exp: -infinity would read as "saw nothing" where results are merged by it."""
    rows = [x + 300 for x in new]
    q, k, v = P._case(new, rows, *SMALL, dtype, 5)
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    n = sum(new)
    q, hit = q[:n].clone(), hit[:n]
    for row, head in ((0, 3), (n - 1, 13)):
        q[row, head, 7] = math.nan
        hit[row, head] = True
    lse = torch.zeros(n, 14, device="cuda")
    ctx = W.Context(W.prefill_workspace_bytes(n, len(new), *SMALL, max(rows), splits))
    out = W.wq_prefill_attention(ctx, q, k, v, R.i32(R.offsets(new)), R.i32(R.offsets(rows)), 0.125, max_kv_rows=max(rows), num_splits=splits, lse=lse)
    _nan_where(out, lse, hit)


@pytest.mark.parametrize("entry", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,own", [((50, 40, 30, 20), None), ((50, 0, 0, 0), (0, 0, 0, 40)), ((0, 0, 0, 0), (0, 0, 0, 40)), ((50, 0, 0, 20), (33, 0, 0, 4))])
def test_a_request_that_is_not_a_number(dtype, lens, own, entry):
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    rng = np.random.default_rng(1)
    prefix = R.make_cache(rng, [lens], 2, 64, 32, t16)[0]
    mine = None if own is None else R.make_cache(rng, [own] * 3, 2, 64, 32, t16)[0]
    q = torch.from_numpy(rng.normal(0, 1, (3, 14, 64))).to(dtype).cuda()
    hit = torch.zeros(3, 14, dtype=torch.bool, device="cuda")
    q[1, 5, 9], hit[1, 5] = entry, True
    lse = torch.zeros(3, 14, device="cuda")
    ctx = W.Context(W.shared_workspace_bytes(3, 1, *SMALL, 200, 100, 2))
    _nan_where(W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, 3]), mine, 0.125, 2, 200, 100, lse=lse), lse, hit)
    if own is not None and not any(own[:3]):
        mine.desc.cap[:] = [0, 0, 0]                     # no room for packed tokens: no launch of their own
        _nan_where(W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, 3]), mine, 0.125, 2, 200, 100, lse=lse), lse, hit)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [(0, 0, 0, 100), (50, 40, 30, 20)])
@pytest.mark.parametrize("plane", ["k16", "v16"])
def test_a_cached_row_that_is_not_a_number(dtype, lens, plane):
    """A key's NaN is every row's of its KV head, a value's that of its channel."""
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    rng = np.random.default_rng(1)
    prefix = R.make_cache(rng, [lens], 2, 64, 32, t16)[0]
    getattr(prefix, plane)[lens[3] - 3, 1, 17] = math.nan
    q = torch.from_numpy(rng.normal(0, 1, (3, 14, 64))).to(dtype).cuda()
    hit = torch.zeros(3, 14, 64, dtype=torch.bool, device="cuda")
    hit[:, 7:, slice(None) if plane == "k16" else 17] = True
    for splits in (1, 3):
        out = W.wq_decode_attention_shared(W.Context(W.shared_workspace_bytes(3, 1, *SMALL, 200, 0, splits)), q, prefix, R.i32([0, 3]), None, 0.125, splits, 200)
        assert torch.equal(out.isnan(), hit)


# ---- values beyond fp16 --------------------------------------------------------------------------------------------------
def _large_rows(g, n, Hkv, hd, dtype):
    return ((torch.rand(n, Hkv, hd, generator=g) + 1) * 2.0 ** 113).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new,splits", [([100], 1), ([100], 2), ([300], 1), ([1], 1), ([1], 3)])
def test_large_values_of_a_prompt(dtype, new, splits):
    """Values below 2^114: 400 weights of up to 2^5 each keep their sums below 2^128."""
    rows = max(new[0], 390)
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn(n, h, 64, generator=g).mul(0.3).to(dtype).cuda() for n, h in ((new[0], 14), (rows, 2)))
    v = _large_rows(g, rows, 2, 64, dtype).cuda()
    ctx = W.Context(W.prefill_workspace_bytes(new[0], 1, *SMALL, rows, splits))
    out = W.wq_prefill_attention(ctx, q, k, v, R.i32([0, new[0]]), R.i32([0, rows]), 0.125, max_kv_rows=rows, num_splits=splits).double().cpu()
    want, lse, spread, terms = R.attend(q.double().cpu(), k.double().cpu(), v.double().cpu(), [rows - new[0] + i + 1 for i in range(new[0])], 0.125)
    w = R.weights_error(rows, 64, terms, float(lse.abs().max()))
    u = R.HALF_STEP[dtype]
    assert bool(((out - want).abs() <= ((0.0 if dtype == torch.float32 else u) + 2 * w) * spread + u * want.abs()).all())


@pytest.mark.parametrize("lens,own", [((0, 0, 0, 200), 0), ((40, 32, 20, 200), 0), ((40, 0, 0, 0), 150), ((0, 33, 0, 100), 150)])
@pytest.mark.parametrize("splits", [1, 3])
def test_large_values_of_shared_caches(lens, own, splits):
    heads, rng, g = SMALL, np.random.default_rng(2), torch.Generator().manual_seed(4)
    prefix, (logical,) = R.make_cache(rng, [lens], 2, 64, 32, torch.bfloat16)
    mine, (own_logical,) = R.make_cache(rng, [(0, 0, 0, own)], 2, 64, 32, torch.bfloat16)
    values = []
    for kv, (k, v), n in ((prefix, logical, lens[3]), (mine, own_logical, own)):
        kv.v16[:n] = _large_rows(g, n, 2, 64, torch.bfloat16).cuda()
        values.append(torch.cat([v[:v.shape[0] - n], kv.v16[:n].double().cpu()]))
    q = torch.from_numpy(rng.normal(0, 0.1, (1, 14, 64))).to(torch.bfloat16).cuda()
    ctx = W.Context(W.shared_workspace_bytes(1, 1, *heads, sum(lens), own, splits))
    out = W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, 1]), mine, 0.125, splits, sum(lens), own).double().cpu()
    k = torch.cat([logical[0], own_logical[0]])
    want, lse, spread, terms = R.attend(q.double().cpu(), k, torch.cat(values), [k.shape[0]], 0.125)
    w = R.weights_error(k.shape[0], 64, terms, float(lse.abs().max()))
    bound = (2 * w + 2.0 ** -8 + math.expm1(2 * 2.0 ** -11 * terms)) * spread + 2.0 ** -8 * want.abs()
    assert bool(((out - want).abs() <= bound).all()), float(((out - want).abs() / bound).max())


# ---- what 16-bit roundings cost -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (SMALL, 64), (LARGE, 32), (LARGE, 64), (LARGE, 128)])
@pytest.mark.parametrize("spread_q", [1.0, 2.0 ** 4])
def test_accuracy_of_16_bit_requests(dtype, heads, group, spread_q):
    """Logits of deviation 3, and of 48 (a peaked softmax whose reference moves).  Roundings are independent, each off by at most half a step (its
    square a third of that squared on the average): of the result; of a weight (fp16 for packed tokens, the rows' type for theirs); of a packed
    value's expansion to fp16 and, for bf16 requests, a key's (fp16 ones meet its codes).  The sum of weights is not rounded, so a weight's rounding acts through its value, a key's through the
    difference from the result.  No element beyond the worst case of all of them, their common size not beyond the mean of the squares."""
    Hq, Hkv, hd = heads
    rng = np.random.default_rng(7)
    lens, own_lens, B, sm, r = (300, 200, 150, 60), (0, 0, 0, 25), 4, 1.0 / math.sqrt(hd), 2.0 ** -11
    prefix, (shared,) = R.make_cache(rng, [lens], Hkv, hd, group, dtype)
    own, mine = R.make_cache(rng, [own_lens] * B, Hkv, hd, group, dtype)
    q = torch.from_numpy(rng.normal(0, 1.3 * spread_q, (B, Hq, hd))).to(dtype).cuda()
    longest = sum(lens)
    ctx = W.Context(W.shared_workspace_bytes(B, 1, *heads, longest, 25))
    lse = torch.empty(B, Hq, device="cuda")
    out = W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, B]), own, sm, 0, longest, 25, lse=lse)
    again = W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, B]), own, sm, 0, longest, 25)
    assert torch.equal(again, out), "two calls differ"
    u = R.HALF_STEP[dtype]
    of_key = r if dtype == torch.bfloat16 else 0.0
    # (a logit's fp32 sums: of codes times scale and of minima, each up to twice the largest minimum beyond the key itself)
    minima = max(float(np.nanmax(np.abs((m[0].cpu().numpy().view(np.uint32) >> 16).astype(np.uint16).view(np.float16).astype(np.float64)))) for m in prefix.meta)
    packed = torch.zeros(longest + 25, dtype=torch.float64)
    packed[:sum(lens[:3])] = 1.0
    off_weight = torch.where(packed > 0, r, u)
    got_all = expected_all = 0.0
    for b in range(B):
        k, v = torch.cat([shared[0], mine[b][0]]), torch.cat([shared[1], mine[b][1]])
        qb = q[b].double().cpu()
        want, want_lse, spread, terms = R.attend(qb[None], k, v, [k.shape[0]], sm)
        want, spread = want[0], spread[0]
        err = (out[b].double().cpu() - want).abs()
        sums = terms + (0.0 if of_key else 2 * minima * float(qb.abs().sum(-1).max()) * sm)
        w, tiny = R.weights_error(k.shape[0], hd, sums, float(want_lse.abs().max())), 2.0 ** -25 if dtype == torch.float16 else 0.0
        bound = (math.expm1(2 * of_key * terms) + 2 * w + u + r) * spread + u * want.abs() + tiny
        assert bool((err <= bound).all()), float((err / bound).max())
        assert bool(((lse[b].double().cpu() - want_lse[0]).abs() <= of_key * terms + 2 * w + 2.0 ** -22 * want_lse[0].abs()).all())
        for h in range(Hq):
            kh, vh = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
            terms_of = qb[h] * kh * sm
            p = torch.softmax(terms_of.sum(1), 0)
            logit = of_key * of_key / 3 * packed * terms_of.square().sum(1)
            var = (u * want[h]).square() / 3 + (p.square()[:, None] * (((off_weight.square() + packed * r * r) / 3)[:, None] * vh.square()
                                                                          + logit[:, None] * (vh - want[h]).square())).sum(0)
            expected_all += float(var.sum())
        got_all += float(err.square().sum())
    assert got_all <= expected_all, math.sqrt(got_all / expected_all)


@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("new,rows,splits", [(130, 600, 1), (9, 600, 3), (2, 600, 1)])
def test_accuracy_of_prompts(dtype, new, rows, splits):
    """As above, with the two roundings that there are: of a weight and of the result."""
    Hq, Hkv, hd = LARGE
    q, k, v = P._case([new], [rows], *LARGE, dtype, 11)
    q = q[:new]
    ctx = W.Context(W.prefill_workspace_bytes(new, 1, *LARGE, rows, splits))
    out = W.wq_prefill_attention(ctx, q, k, v, R.i32([0, new]), R.i32([0, rows]), 1 / math.sqrt(hd), max_kv_rows=rows, num_splits=splits).double().cpu()
    qd, kd, vd = q.double().cpu(), k[:rows].double().cpu(), v[:rows].double().cpu()
    limit = [rows - new + i + 1 for i in range(new)]
    want = R.attend(qd, kd, vd, limit, 1 / math.sqrt(hd))[0]
    u = R.HALF_STEP[dtype]
    expected = (u * want).square().sum() / 3
    hidden = torch.arange(rows)[None] >= torch.tensor(limit)[:, None]
    for h in range(Hq):
        s = qd[:, h] @ kd[:, h // (Hq // Hkv)].T / math.sqrt(hd)
        p = torch.softmax(s.masked_fill(hidden, -math.inf), 1)
        expected += (p.square() @ vd[:, h // (Hq // Hkv)].square()).sum() * u * u / 3
    assert float((out - want).square().sum()) <= float(expected), math.sqrt(float((out - want).square().sum() / expected))
