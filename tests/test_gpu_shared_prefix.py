"""Decode attention of requests that share packed caches, against plain attention in 64 bits over the same values."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
SMALL, LARGE = (14, 2, 64), (28, 4, 128)


def _check(prefixes, groups, own_lens, heads, group, dtype, splits=0, front=0, seed=1, scale=1.0, spread_q=1.0):
    """prefixes[p] = tokens per class; groups[p] = its requests; `front` requests lie in front of the first group."""
    Hq, Hkv, hd = heads
    rng = np.random.default_rng(seed)
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    prefix, shared = R.make_cache(rng, prefixes, Hkv, hd, group, t16, scale=scale)
    off = [front + x for x in R.offsets(groups)]
    B = len(own_lens) if own_lens is not None else off[-1]
    own, mine = R.make_cache(rng, own_lens, Hkv, hd, group, t16, slack=3, scale=scale) if own_lens is not None else (None, [(torch.zeros(0, Hkv, hd).double(),) * 2] * B)
    q = torch.from_numpy(rng.normal(0, 2.0 / (scale * 1.5) * spread_q, (B, Hq, hd))).to(dtype).cuda()
    sm = 1.0 / math.sqrt(hd)
    longest = max([sum(p) for p in prefixes] + [0])
    longest_own = max(sum(x) for x in own_lens) if own_lens is not None else 0
    ctx = W.Context(W.shared_workspace_bytes(B, len(prefixes), Hq, Hkv, hd, longest, longest_own, splits))
    lse = torch.empty(B, Hq, device="cuda")
    out = W.wq_decode_attention_shared(ctx, q, prefix, R.i32(off), own, sm, splits, longest, longest_own, lse=lse)
    assert out.dtype == dtype
    u = R.HALF_STEP[dtype]
    exact = dtype == torch.float32
    num = den = 0.0
    for b in range(B):
        p = next((i for i in range(len(groups)) if off[i] <= b < off[i + 1]), None)
        parts = ([shared[p]] if p is not None else []) + [mine[b]]
        k, v = torch.cat([x[0] for x in parts]), torch.cat([x[1] for x in parts])
        want, want_lse, spread, terms = (x[0] if torch.is_tensor(x) else x for x in R.attend(q[b:b + 1].double().cpu(), k, v, [k.shape[0]], sm))
        got, got_lse = out[b].double().cpu(), lse[b].double().cpu()
        if k.shape[0] == 0:
            assert bool((got == 0).all()) and bool((got_lse == -math.inf).all())
            continue
        w = R.weights_error(k.shape[0], hd, terms, float(want_lse.abs().max()))
        # 16-bit queries: keys, values and weights each rounded to 11 bits (keys: of every product of a logit), bf16 rows' weights to 8; the
        # requests' own caches within the decode kernel's 2e-3 of the vector's largest entry
        soft = 0.0 if exact else 2.0 ** -11 * terms + u + 2 * 2.0 ** -11
        bound = (2 * w + soft) * spread + u * want.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
        if not exact:
            bound = bound + 2.0 ** -11 * terms * want.abs() + 2e-3 * spread.amax(-1, keepdim=True) + 2.0 ** -35 * v.abs().sum(0).repeat_interleave(Hq // Hkv, 0)
        err = (got - want).abs()
        assert bool((err <= bound).all()), (b, float((err / bound).max()))
        assert bool(((got_lse - want_lse).abs() <= 2 * w + 2.0 ** -22 * want_lse.abs() + (0.0 if exact else 2.0 ** -11 * terms + 2e-3)).all())
        num, den = num + float(err.square().sum()), den + float(want.square().sum())
    # roundings are independent: their common size is well below the bound of the worst case.  Output and weights at u (rms u / sqrt 3 each),
    # values at 2^-11, a logit of deviation 2 by 2^-11 of its terms
    if den and not exact:
        assert math.sqrt(num / den) <= 1.5 * u + 6 * 2.0 ** -11, math.sqrt(num / den)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (SMALL, 64), (LARGE, 64), (LARGE, 32), (LARGE, 128), ((8, 8, 64), 32), ((16, 2, 128), 64)])
def test_mixed_prefix(dtype, heads, group):
    _check([(100, 64, 33, 20)], [3], [(0, 0, 0, 5), (0, 0, 0, 1), (0, 0, 0, 40)], heads, group, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens", [(1, 0, 0, 0), (0, 31, 0, 0), (0, 0, 65, 0), (0, 0, 0, 1), (0, 0, 0, 200), (33, 0, 0, 64), (0, 0, 0, 0)])
@pytest.mark.parametrize("splits", [1, 5])
def test_single_classes_and_tiny_prefixes(dtype, lens, splits):
    _check([lens], [2], None, SMALL, 32, dtype, splits)
    _check([lens], [2], [(0, 0, 0, 3), (0, 0, 0, 0)], LARGE, 64, dtype, splits)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_groups(dtype):
    # groups of none, one and more requests than a workgroup has rows for; requests in front of and behind all groups; own caches packed too
    prefixes = [(32, 0, 7, 3), (0, 0, 0, 0), (70, 130, 10, 0), (5, 5, 5, 5)]
    groups = [0, 4, 21, 1]
    own = [(40 if b % 5 == 0 else 0, 0, 9 if b % 7 == 1 else 0, b % 4 * 11) for b in range(2 + 26 + 3)]
    _check(prefixes, groups, own, SMALL, 32, dtype, front=2)
    _check(prefixes, groups, own, LARGE, 64, dtype, 3, front=2, seed=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale,spread_q", [(2.0 ** -6, 1.0), (2.0 ** 5, 1.0), (1.0, 2.0 ** 4)])
def test_magnitudes(dtype, scale, spread_q):
    if spread_q == 1.0:
        _check([(64, 96, 40, 30)], [2], [(0, 0, 0, 8)] * 2, LARGE, 64, dtype, scale=scale)
    else:                                                         # a peaked softmax; the statistical part of the check is for logits of deviation 2
        _check([(64, 96, 40, 30)], [2], [(0, 0, 0, 8)] * 2, SMALL, 32, torch.float32, scale=scale, spread_q=spread_q)


def test_long_prefix():
    _check([(2500, 2000, 1100, 150)], [40], [(0, 0, 0, 3 + b) for b in range(40)], (14, 2, 128), 64, torch.bfloat16)
    _check([(700, 0, 1100, 1250)], [3], None, SMALL, 64, torch.float16)


@pytest.mark.parametrize("own_len", [(0, 0, 0, 3000), (1000, 700, 500, 40)])
def test_long_own_caches(own_len):
    """Beyond the length up to which they are part of the shared launch, and just below."""
    for dtype in DTYPES:
        _check([(64, 0, 40, 30)], [2], [own_len, (0, 0, 0, 9)], SMALL, 32, dtype)
    _check([(64, 0, 40, 30)], [1], [tuple(x * 2048 // 3000 for x in own_len)], LARGE, 64, torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_own_rows_of_many_requests(dtype):
    """Enough requests to fill the card: their own rows are walked beside the merge whatever their number."""
    own = [(0, 0, 0, 1100 if b % 31 == 0 else b % 7) for b in range(65)]
    _check([(64, 0, 40, 30), (0, 32, 0, 3)], [60, 5], own, (8, 4, 64), 32, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_segment_far_into_its_buffers(dtype):
    """8-bit codes and 16-bit rows of which the last ones are used: 5.2 GB of codes, 4.3 GB of rows."""
    heads, hd, t16 = (8, 2, 64), 64, torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    near, _ = R.make_cache(np.random.default_rng(5), [(0, 0, 190, 77)], 2, hd, 32, t16)
    far16, far = 1 << 24, 20480000
    wide = W.PackedKV(1, 2, hd, 32, t16, [0, 0, far + near.cap[2]], [far16, far16 + 77])
    wide.codes[2][:, :, far * hd:] = near.codes[2]
    wide.meta[2][:, :, far * 2:] = near.meta[2]
    wide.cls_off[2].copy_(near.cls_off[2] + far)
    wide.cls_len[2].copy_(near.cls_len[2])
    wide.k16[far16:], wide.v16[far16:] = near.k16, near.v16
    wide.len16.copy_(near.len16)
    q = torch.randn(3, 8, hd, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    own, _ = R.make_cache(np.random.default_rng(6), [(0, 0, 0, 40)], 2, hd, 32, t16)
    ctx = W.Context(W.shared_workspace_bytes(3, 1, *heads, 300, 100))
    req = R.i32([0, 3])
    a = [W.wq_decode_attention_shared(ctx, q, x, req, None, 0.1, 2, 300) for x in (near, wide)]
    assert torch.equal(a[0], a[1]) and bool(a[0].isfinite().all())
    # ... and as a request's own rows
    for x in (near, wide):
        x.cls_len[2].zero_()
        x.desc.cap[:] = [0, 0, 0]                # no room for packed tokens
    b = [W.wq_decode_attention_shared(ctx, q[:1], own, R.i32([0, 1]), x, 0.1, 2, 300, 77) for x in (near, wide)]
    assert torch.equal(b[0], b[1]) and bool(b[0].isfinite().all())


@pytest.mark.parametrize("bits", [2, 4, 8])
def test_values_at_the_end_of_fp16(bits):
    """A group from -65504 to 65504: the rounded scale carries its largest code past fp16's range, where the result is fp16's largest value."""
    hd, Hkv, n, c = 64, 1, 32, {2: 0, 4: 1, 8: 2}[bits]
    top = 2 ** bits - 1
    s = np.float16((65504.0 + 65504.0) / top)
    assert -65504.0 + float(s) * top >= 65520.0 or bits == 8
    for dtype in (torch.float16, torch.bfloat16):
        kv = W.PackedKV(1, Hkv, hd, 32, dtype, [n if i == c else 0 for i in range(3)], [0, 0], fill=0)
        kv.codes[c].fill_(255)                                              # every code the largest one
        kv.meta[c].fill_(int(np.uint32(np.float16(s).view(np.uint16)) | np.uint32(np.float16(-65504).view(np.uint16)) << 16) - (1 << 32))
        kv.meta[c][0].zero_()                                               # keys of zero
        kv.cls_off[c].copy_(R.i32([0, n]))
        kv.cls_len[c].copy_(R.i32([n]))
        ctx = W.Context(W.shared_workspace_bytes(1, 1, 1, 1, hd, n))
        q = torch.ones(1, 1, hd, dtype=dtype, device="cuda")
        out = W.wq_decode_attention_shared(ctx, q, kv, R.i32([0, 1]), None, 0.125).float()
        want = min(-65504.0 + float(s) * top, 65504.0)
        assert bool(((out - want).abs() <= 2 * R.HALF_STEP[dtype] * want).all()), (dtype, out.min(), out.max(), want)


def test_bf16_queries_beyond_fp16():
    """A bf16 query's magnitude has no bound of fp16's: the result is that of the scaled query and the inverse softmax scale."""
    rng = np.random.default_rng(0)
    prefix, _ = R.make_cache(rng, [(50, 40, 30, 20)], 4, 128, 64, torch.bfloat16)
    q = torch.from_numpy(rng.normal(0, 1, (2, 28, 128))).to(torch.bfloat16).cuda()
    ctx = W.Context(W.shared_workspace_bytes(2, 1, 28, 4, 128, 140))
    for e in (-60, 60):
        big = (q.double() * 2.0 ** e).to(torch.bfloat16)
        a = W.wq_decode_attention_shared(ctx, q, prefix, R.i32([0, 2]), None, 0.125)
        b = W.wq_decode_attention_shared(ctx, big, prefix, R.i32([0, 2]), None, 0.125 * 2.0 ** -e)
        assert torch.equal(a, b)


def test_captured_decode_steps_grow_their_own_caches():
    """The operators as a program uses them: rotary positions and prompt attention, the prompt packed, then captured steps of rotary append and
    shared decode for three questions about it."""
    Hq, Hkv, hd, win, nwin, text = 14, 2, 64, 16, 8, 19
    rows = win * nwin + text
    g = torch.Generator().manual_seed(0)
    qkv = torch.randn(rows, (Hq + 2 * Hkv) * hd, generator=g).to(torch.bfloat16).cuda()
    cut = lambda a, z: qkv[:, a * hd:z * hd].unflatten(-1, (-1, hd))  # noqa: E731
    inv_freq = torch.tensor(W.wq_rope_frequencies(hd, 1000000.0)[0]).cuda()
    sm = 1.0 / math.sqrt(hd)
    B = 3
    need = max(W.prefill_workspace_bytes(rows, 1, Hq, Hkv, hd, rows), W.shared_workspace_bytes(B, 1, Hq, Hkv, hd, rows, 8))
    stream = torch.cuda.Stream()
    ctx = W.Context(need, stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        q, k = W.wq_rope(ctx, cut(0, Hq), cut(Hq, Hq + Hkv), torch.arange(rows, dtype=torch.int32, device="cuda"), inv_freq)
        v = cut(Hq + Hkv, Hq + 2 * Hkv).contiguous()
        off = R.i32([0, rows])
        W.wq_prefill_attention(ctx, q, k, v, off, off, sm, R.i32([win * nwin]), rows)
        scores = torch.linspace(1, 0, nwin, device="cuda")
        bits, perm, seg = W.wq_assign_bits(ctx, scores, R.i32([0, nwin]), nwin, quota=torch.tensor([[2, 3, 3]], dtype=torch.int32, device="cuda"))
        prefix = W.PackedKV(1, Hkv, hd, 32, torch.bfloat16, [3 * win + 32, 3 * win + 32, 2 * win], [0, text])
        W.wq_reorder_quantize(ctx, k, v, off, R.i32([win]), R.i32([0, nwin]), perm, seg, rows, prefix)
        own = W.PackedKV(B, Hkv, hd, 32, torch.bfloat16, [0, 0, 0], [0, 8, 16, 24])
        qn, kn, vn = (torch.randn(B, h, hd, generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
        pos = torch.full((B,), rows, dtype=torch.int32, device="cuda")
        req = R.i32([0, B])
        turned, out = torch.empty_like(qn), torch.empty_like(qn)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            W.wq_rope_append_kv(ctx, qn, kn, vn, pos, inv_freq, own, q_out=turned)
            W.wq_decode_attention_shared(ctx, turned, prefix, req, own, sm, 0, rows, 8, out=out)
            pos.add_(1)
            qn.mul_(-1)
        dense = W.PackedKV(1, Hkv, hd, 32, torch.bfloat16, [0, 0, 0], [0, rows])
        W.wq_dequantize(ctx, prefix, dense)
        torch.cuda.synchronize()
        kk, vv = dense.k16.double().cpu(), dense.v16.double().cpu()
        for step in range(5):
            query = (qn.clone()).double().cpu()
            graph.replay()
            torch.cuda.synchronize()
            assert own.len16.tolist() == [step + 1] * B
            wq = R.rope(query, torch.full((B,), rows + step), inv_freq.cpu(), W.ROPE_HALF, 1.0)[0]
            for b in range(B):
                n = 8 * b + step + 1
                ko, vo = own.k16[8 * b:n].double().cpu(), own.v16[8 * b:n].double().cpu()
                want = R.attend(wq[b:b + 1], torch.cat([kk, ko]), torch.cat([vv, vo]), [rows + step + 1], sm)[0][0]
                # (the dequantized copy is rounded to bf16: 2^-8 of a value, in 64 channels of a logit of deviation 1)
                assert float((out[b].double().cpu() - want).norm() / want.norm()) <= 2e-2
        assert ctx.device_status() == 0
