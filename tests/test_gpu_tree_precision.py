"""What attention of several new rows per sequence may lose to roundings, kernel by kernel: the log-sum-exp of 16-bit queries, results as a whole, softmaxes of one key; and
entries that are not finite.  rows new rows of 7 heads a KV head are 14, 28, 42 and 140 query rows: tiles of 16, 32, 48 and 128 of them in 16-bit types."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import tree_ref as T
from tests.test_gpu_tree_attention import DTYPES, LARGE, SMALL, _inputs

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]
ROWS = [2, 4, 6, 20]


class _Call:
    """A batch of random trees and its 64-bit logical contents."""

    def __init__(self, lens, rows, heads, group, dtype, seed=1, spread_q=1.0, keys=True):
        self.rng, self.dtype, self.rows, self.sm = np.random.default_rng(seed), dtype, rows, 1.0 / math.sqrt(heads[2])
        self.Hq, self.Hkv, self.hd = heads
        self.lens, self.kv, self.cached = lens, *R.make_cache(self.rng, lens, self.Hkv, self.hd, group, torch.bfloat16 if dtype == torch.bfloat16 else torch.float16)
        self.q, self.k, self.v = _inputs(self.rng, rows * len(lens), heads, dtype, spread_q=spread_q)
        if not keys:
            self.k.zero_()
        self.parents = [T.random_tree(self.rng, rows) for _ in lens]

    def run(self, splits=0, with_lse=True):
        n, B, longest = self.rows * len(self.lens), len(self.lens), max(sum(x) for x in self.lens)
        ctx = W.Context(W.tree_workspace_bytes(n, B, self.Hq, self.Hkv, self.hd, longest, self.rows, splits))
        lse = torch.full((n, self.Hq), 77.0, device="cuda") if with_lse else None
        out = W.wq_tree_attention(ctx, self.q, self.k, self.v, self.kv, R.i32([self.rows * i for i in range(B + 1)]), self.sm, R.i32(sum(self.parents, [])), self.rows, longest, splits,
                                  lse=lse)
        assert ctx.device_status() == 0
        return out, lse

    def sequence(self, b):
        """(slice of its rows, queries, keys, values, who sees whom), in 64 bits."""
        s = slice(self.rows * b, self.rows * (b + 1))
        kk, vv = (torch.cat([c, x[s].double().cpu()]) for c, x in zip(self.cached[b], (self.k, self.v)))
        sees = torch.cat([torch.ones(self.rows, self.cached[b][0].shape[0], dtype=torch.bool), T.seen(self.parents[b], self.rows)], 1)
        return s, self.q[s].double().cpu(), kk, vv, sees

    def code_sizes(self, b):
        """[keys, Hkv, hd]: the magnitudes that a key's channel is made of, |scale code| + |minimum| (a plain row's: the entry)."""
        c64 = self.cached[b][0].abs()
        at = 0
        for c in range(3):
            G, n, first = self.hd // self.kv.group, int(self.kv.cls_len[c][b]), int(self.kv.cls_off[c][b])
            words = self.kv.meta[c][0].cpu().view(self.Hkv, -1, G, 16).permute(1, 3, 0, 2).reshape(-1, self.Hkv, G)[first:first + n]
            m = (words >> 16).to(torch.int16).view(torch.float16).double().abs().repeat_interleave(self.kv.group, -1)
            c64[at:at + n] += 2 * m                                      # |s c| <= |s c + m| + |m|
            at += n
        return torch.cat([c64, self.k[self.rows * b:self.rows * (b + 1)].double().cpu().abs()])


def _rms(x):
    return float(torch.cat([y.flatten() for y in x]).square().mean().sqrt())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (SMALL, 64), (LARGE, 32), (LARGE, 64), (LARGE, 128)])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("splits", [1, 2])
def test_log_sum_exp_of_packed_keys(dtype, heads, group, rows, splits):
    """Packed keys enter the logits of a call with lse as codes, a group's scale and minimum in fp32: additions of fp32, each off by 2^-24 of a partial sum (2^-23 with
    the instruction's own sums), are all that lse loses.  They are independent, and a partial sum is at most what the key's magnitudes make: hd of them, 8 for
    scales, minima, exponent, sums.  Keys rounded to fp16 would be off by more: that is computed here, and has to lie outside of the bound."""
    call = _Call([(0, 0, 5, 0), (0, 0, 3, 0), (0, 0, 8, 0)], rows, heads, group, dtype, seed=rows, keys=False)
    lse = call.run(splits)[1]
    errors, rounded, sizes, values = [], [], [], []
    for b in range(3):
        s, q, kk, vv, sees = call.sequence(b)
        want = T.attend(q, kk, vv, sees, call.sm)[1]
        rounded.append(T.attend(q, kk.half().double(), vv, sees, call.sm)[1] - want)
        size = call.code_sizes(b).repeat_interleave(call.Hq // call.Hkv, 1)
        sizes.append(torch.einsum("nhc,thc->nht", q.abs(), size).amax(-1) * call.sm)
        errors.append(lse[s].double().cpu() - want)
        values.append(want)
    bound = math.sqrt(call.hd + 8) * 2.0 ** -23 * _rms(sizes) + 2.0 ** -22 * _rms(values)
    assert _rms(rounded) > 2 * bound, (_rms(rounded), bound)
    assert _rms(errors) <= bound, (_rms(errors), bound, _rms(rounded))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("heads,group", [(SMALL, 32), (LARGE, 64)])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("with_lse", [False, True])
def test_results_as_a_whole(dtype, heads, group, rows, with_lse):
    """A rounding to nearest has a common size of half a step / sqrt 3.  The result has one, the weights one of the values' type, packed values one to 11 bits, and so have
    their weights; packed keys one of 11 bits without lse in bf16, in logits of deviation 2.  Independent, their squares add up; a twentieth more for the sample."""
    call = _Call([(100, 64, 33, 20), (0, 40, 0, 3), (70, 0, 90, 0)], rows, heads, group, dtype, seed=rows)
    out = call.run(0, with_lse)[0]
    err, size = [], []
    for b in range(3):
        s, q, kk, vv, sees = call.sequence(b)
        want = T.attend(q, kk, vv, sees, call.sm)[0]
        err.append(out[s].double().cpu() - want)
        size.append(want)
    u, f = R.HALF_STEP[dtype] / math.sqrt(3), 2.0 ** -11 / math.sqrt(3)
    keys = 2 * f if dtype == torch.bfloat16 and not with_lse else 0.0
    assert _rms(err) / _rms(size) <= 1.05 * math.sqrt(2 * u ** 2 + f ** 2 + keys ** 2), _rms(err) / _rms(size)


def _bound(call, b, q, kk, vv, spread, want, want_lse, rounded_keys):
    """Of a result's error and a log-sum-exp's.  A logit is off by w (fp32) and, where keys are rounded, by 2^-11 of the sum of its terms' magnitudes; every weight and
    their sum by that much of themselves; then the roundings of a weight, a packed value and the result."""
    size = call.code_sizes(b)[:kk.shape[0]].repeat_interleave(call.Hq // call.Hkv, 1)
    terms = float((torch.einsum("nhc,thc->nht", q.abs().nan_to_num(0, 0, 0), size.nan_to_num(0, 0, 0)) * call.sm).max())
    finite = want_lse[want_lse.isfinite()].abs()
    w = R.weights_error(kk.shape[0], call.hd, terms, float(finite.max()) if finite.numel() else 0.0)
    logit = w + (2.0 ** -11 * terms if rounded_keys else 0.0)
    exact, u = call.dtype == torch.float32, R.HALF_STEP[call.dtype]
    # weights below a type's range are lost: 2^-35 of the largest in fp16, 2^-120 (and results below 2^-126) in fp32
    lost = 2.0 ** (-120 if exact else -35) * vv.abs().nan_to_num(0, 0, 0).sum(0).repeat_interleave(call.Hq // call.Hkv, 0)
    factor = (1 + math.expm1(2 * logit)) * (1 + u) * (1 + (u if exact else 2.0 ** -11)) - 1
    bound = (factor * spread + lost) * (1 + u) + u * want.abs() + (2.0 ** -126 if exact else 2.0 ** -25 if call.dtype == torch.float16 else 0.0)
    return bound, logit + 2.0 ** -22 * want_lse.abs()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("splits", [1, 3])
def test_softmaxes_of_one_key(dtype, rows, splits):
    """Logits of deviation 32: the references move again and again, most weights are lost."""
    for heads, group in ((SMALL, 32), (LARGE, 64)):
        call = _Call([(100, 64, 33, 20), (0, 40, 0, 3), (7, 0, 90, 0)], rows, heads, group, dtype, seed=rows, spread_q=16.0)
        for with_lse in (False, True):
            out, lse = call.run(splits, with_lse)
            for b in range(3):
                s, q, kk, vv, sees = call.sequence(b)
                want, want_lse, spread, _ = T.attend(q, kk, vv, sees, call.sm)
                bound, bound_lse = _bound(call, b, q, kk, vv, spread, want, want_lse, dtype == torch.bfloat16 and not with_lse)
                err = (out[s].double().cpu() - want).abs()
                assert bool((err <= bound).all()), float((err / bound).max())
                if with_lse:
                    err = (lse[s].double().cpu() - want_lse).abs()
                    assert bool((err <= bound_lse).all()), float((err / bound_lse).max())


def _check_finite_and_not(call, out, lse, b, nowhere, rounded_keys):
    """Rows of `nowhere` [rows, Hq] are NaN, their lse not finite; the others are what 64 bits say."""
    s, q, kk, vv, sees = call.sequence(b)
    want, want_lse, spread, _ = T.attend(q, kk, vv, sees, call.sm)
    assert bool((want.isnan().all(-1) == nowhere).all()) and bool((want.isnan().any(-1) == nowhere).all())
    got, got_lse = out[s].double().cpu(), None if lse is None else lse[s].double().cpu()
    assert bool(got[nowhere].isnan().all()) and (lse is None or not bool(got_lse[nowhere].isfinite().any()))
    bound, bound_lse = _bound(call, b, q, kk, vv, spread, want, want_lse, rounded_keys)
    assert bool(((got - want).abs() <= bound)[~nowhere].all()) and (lse is None or bool(((got_lse - want_lse).abs() <= bound_lse)[~nowhere].all()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_queries_that_are_not_finite(dtype, rows, splits, value):
    """NaN and infinity in one row's query (keys of both signs: a product is +infinity), over packed tokens, plain rows and new rows alone."""
    for heads, group in ((SMALL, 32), (LARGE, 64)):
        call = _Call([(64, 40, 33, 20), (0, 0, 0, 50), (0, 70, 0, 0)], rows, heads, group, dtype, seed=rows)
        nowhere = torch.zeros(rows, call.Hq, dtype=torch.bool)
        nowhere[rows - 1, 5] = True
        for b in range(3):
            call.q[rows * b + rows - 1, 5, 9] = value
        for with_lse in (False, True):
            out, lse = call.run(splits, with_lse)
            for b in range(3):
                _check_finite_and_not(call, out, lse, b, nowhere, dtype == torch.bfloat16 and not with_lse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_keys_that_are_not_finite(dtype, rows, splits, value):
    """... in the key of a new row: the rows that see it have a logit of NaN or infinity (a weight of zero for -infinity), the others do not know of it."""
    for heads, group in ((SMALL, 32), (LARGE, 64)):
        call = _Call([(64, 40, 33, 20), (0, 0, 0, 50), (0, 0, 0, 0)], rows, heads, group, dtype, seed=rows)
        for b in range(3):
            call.k[rows * b + rows // 2, 1, 7] = value
        for with_lse in (False, True):
            out, lse = call.run(splits, with_lse)
            for b in range(3):
                s, q, kk, vv, sees = call.sequence(b)
                at = kk.shape[0] - rows + rows // 2
                logit = q[:, :, 7] * value
                nowhere = sees[:, at][:, None] & (logit.isnan() | (logit == math.inf))
                nowhere[:, :call.Hq // call.Hkv] = False                 # (the other KV heads' keys are finite)
                nowhere[:, 2 * (call.Hq // call.Hkv):] = False
                _check_finite_and_not(call, out, lse, b, nowhere, dtype == torch.bfloat16 and not with_lse)
