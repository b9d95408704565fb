"""Refusals and host helpers of the operators around the cache: reported before anything is enqueued, so no GPU is needed."""
import ctypes as C
import math
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def W():
    if not os.path.exists(os.path.join(ROOT, "paper_2605_02262_amd", "libwq.so")):
        from paper_2605_02262_amd import build
        build.build(verbose=False)
    from paper_2605_02262_amd import binding
    return binding


@pytest.fixture
def ctx(W):
    h = C.c_void_p()
    assert W.lib().wq_create(C.byref(h), None, C.c_void_p(0x10000), 1 << 20) == 0     # never dereferenced
    yield h
    W.lib().wq_destroy(h)


P = 0x1000          # a pointer that nothing follows
BF, F32 = 1, 0


def _rope(W, ctx, **more):
    a = dict(q=P, qs=14 * 64, k=P, ks=128, dtype=BF, rows=0x7fffffff, Hq=14, Hkv=2, hd=64, rot=64, layout=0, pos=P, inv=P, m=1.0, qo=2 * P, qos=14 * 64, ko=3 * P, kos=128)
    a.update(more)
    return W.lib().wq_rope(ctx, a["q"], a["qs"], a["k"], a["ks"], a["dtype"], a["rows"], a["Hq"], a["Hkv"], a["hd"], a["rot"], a["layout"], a["pos"], a["inv"], a["m"],
                           a["qo"], a["qos"], a["ko"], a["kos"])


@pytest.mark.parametrize("bad,code", [
    (dict(hd=96), -2), (dict(rot=0), -2), (dict(rot=24), -2), (dict(rot=80), -2), (dict(dtype=7), -1), (dict(layout=2), -1), (dict(rows=-1), -1), (dict(rows=1 << 31), -2),
    (dict(Hq=0), -1), (dict(Hkv=-1), -1), (dict(Hq=1 << 17), -2), (dict(q=None), -1), (dict(k=None), -1), (dict(qo=None), -1), (dict(ko=None), -1), (dict(pos=None), -1),
    (dict(inv=None), -1), (dict(qs=14 * 64 - 8), -1), (dict(qs=14 * 64 + 4), -1), (dict(q=P + 8), -1), (dict(qo=P + 2), -1), (dict(kos=64), -1), (dict(m=math.nan), -1),
    (dict(m=math.inf), -1), (dict(qo=P, qos=2048), -1), (dict(ko=P, kos=2048), -1)])
def test_rope_refuses(W, ctx, bad, code):
    assert _rope(W, ctx, **bad) == code
    assert W.lib().wq_last_error(ctx)


def test_rope_of_no_rows(W, ctx):
    assert _rope(W, ctx, rows=0) == 0 and _rope(W, ctx, rows=0, q=None, k=None, pos=None, inv=None, qo=None, ko=None) == 0
    assert W.lib().wq_rope(None, *([None, 0] * 2), 0, 0, 1, 0, 64, 64, 0, None, None, 1.0, None, 0, None, 0) == -1


def _desc(W, B=2, Hkv=2, hd=64, group=32, dtype16=1, cap16=64):
    d = W._PackedKV()
    d.B, d.Hkv, d.hd, d.group, d.dtype16, d.cap16 = B, Hkv, hd, group, dtype16, cap16
    for c in range(3):
        d.codes[c], d.meta[c], d.cap[c], d.cls_off[c], d.cls_len[c] = P, P, 64, P, P
    d.k16 = d.v16 = d.off16 = d.len16 = d.v_scale_max = P
    return d


def test_rope_append_refuses(W, ctx):
    def call(d, **more):
        a = dict(dtype=BF, B=2, rot=64, q=P, qo=2 * P, v=P, vs=128)
        a.update(more)
        return W.lib().wq_rope_append_kv(ctx, a["q"], 14 * 64, P, 128, a["v"], a["vs"], a["dtype"], a["B"], 14, a["rot"], 0, P, P, 1.0, a["qo"], 14 * 64,
                                         None if d is None else C.byref(d))
    assert call(None) == -1 and call(_desc(W, B=3)) == -1 and call(_desc(W, hd=96)) == -2 and call(_desc(W), rot=128) == -2
    assert call(_desc(W), dtype=2) == -1 and call(_desc(W, dtype16=2)) == -1 and call(_desc(W), dtype=F32) == -1
    assert call(_desc(W), v=None) == -1 and call(_desc(W), v=P + 4) == -1 and call(_desc(W), vs=64) == -1 and call(_desc(W), qo=None) == -1
    d = _desc(W)
    d.k16 = P + 2
    assert call(d) == -1
    assert call(_desc(W, B=0), B=0) == 0 and call(_desc(W), B=-1) == -1


def _prefill(W, ctx, **more):
    a = dict(q=P, qs=14 * 64, k=P, ks=128, v=P, vs=128, dtype=BF, B=2, Hq=14, Hkv=2, hd=64, qo=P, ko=P, pre=None, tq=100, tk=100, mk=100, sm=0.125, splits=1, out=P, lse=None)
    a.update(more)
    return W.lib().wq_prefill_attention(ctx, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], a["B"], a["Hq"], a["Hkv"], a["hd"], a["qo"], a["ko"], a["pre"],
                                        a["tq"], a["tk"], a["mk"], a["sm"], a["splits"], a["out"], a["lse"])


@pytest.mark.parametrize("bad,code", [
    (dict(B=-1), -1), (dict(tq=-1), -1), (dict(tk=-1), -1), (dict(dtype=3), -1), (dict(hd=256), -2), (dict(Hq=15), -2), (dict(Hq=18, qs=18 * 64), -2), (dict(Hkv=0), -2),
    (dict(tq=1 << 31), -2), (dict(tk=1 << 31), -2), (dict(splits=-1), -1), (dict(splits=65), -1), (dict(sm=0.0), -1), (dict(sm=math.nan), -1), (dict(sm=math.inf), -1),
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(qo=None), -1), (dict(ko=None), -1), (dict(out=None), -1), (dict(out=P + 8), -1), (dict(q=P + 8), -1),
    (dict(qs=100), -1), (dict(ks=132), -1), (dict(vs=64), -1), (dict(splits=64), -4), (dict(tq=1000000, splits=2), -4),
    (dict(B=5000000), -2), (dict(tq=1 << 27, Hq=1, Hkv=1, splits=2), -2)])
def test_prefill_refuses(W, ctx, bad, code):
    assert _prefill(W, ctx, **bad) == code
    assert W.lib().wq_last_error(ctx)


def test_prefill_of_nothing(W, ctx):
    assert _prefill(W, ctx, B=0) == 0 and _prefill(W, ctx, tq=0) == 0 and _prefill(W, None) == -1


def test_shared_refuses(W, ctx):
    def call(prefix, own, **more):
        a = dict(q=P, dtype=BF, B=2, Hq=14, req=P, sm=0.125, splits=1, out=P)
        a.update(more)
        return W.lib().wq_decode_attention_shared(ctx, a["q"], a["dtype"], a["B"], a["Hq"], None if prefix is None else C.byref(prefix), a["req"],
                                                  None if own is None else C.byref(own), a["sm"], a["splits"], 100, 100, a["out"], None)
    ok = lambda **k: _desc(W, **k)  # noqa: E731
    assert call(None, None) == -1 and call(ok(hd=32), None) == -2 and call(ok(dtype16=0), None) == -1
    assert call(ok(), None, dtype=2) == -1 and call(ok(dtype16=2), None) == -1 and call(ok(), None, dtype=F32) == -1 and call(ok(), None, dtype=9) == -1
    assert call(ok(), None, Hq=15) == -2 and call(ok(), None, Hq=18) == -2 and call(ok(), None, Hq=0) == -1 and call(ok(), None, B=-1) == -1 and call(ok(), None, B=65536) == -2
    assert call(ok(), None, q=P + 8) == -1 and call(ok(), None, out=P + 8) == -1 and call(ok(), None, q=None) == -1 and call(ok(), None, out=None) == -1
    assert call(ok(), None, req=None) == -1 and call(ok(), None, splits=65) == -1 and call(ok(), None, splits=-1) == -1 and call(ok(), None, sm=-1.0) == -1
    assert call(ok(), ok(B=3)) == -1 and call(ok(), ok(hd=128, group=64)) == -1 and call(ok(), ok(Hkv=1)) == -1 and call(ok(), ok(dtype16=2)) == -1
    for field in ("k16", "v16"):
        d = ok()
        setattr(d, field, P + 8)
        assert call(d, None) == -1
    d = ok()
    d.codes[1] = P + 4
    assert call(d, None) == -1
    assert call(ok(), None, splits=64, B=1000) == -4 and call(ok(B=65536), None) == -2 and call(ok(B=0), None) == -1
    assert call(ok(), ok(B=0), B=0) == 0


def test_workspace_helpers(W):
    assert W.prefill_workspace_bytes(100, 1, 28, 4, 128, 100, 1) == 16384
    assert W.prefill_workspace_bytes(100, 1, 28, 4, 128, 100, 8) >= 16384 + 100 * 28 * 8 * 130 * 4
    assert W.prefill_workspace_bytes(0, 1, 28, 4, 128, 100) == 16384 and W.prefill_workspace_bytes(1, 1, 28, 3, 128, 100) == 16384
    assert W.shared_workspace_bytes(4, 1, 28, 4, 128, 50000, 100, 8) >= 16384 + 4 * 28 * (8 * 130 + 129) * 4
    assert W.shared_workspace_bytes(0, 1, 28, 4, 128, 50000, 100) == 16384
    for total_q in (1, 7, 300, 100000):
        for longest in (1, 64, 5000, 1000000):
            assert W.prefill_workspace_bytes(total_q, 3, 28, 4, 128, longest) <= 16384 + total_q * 28 * 64 * 130 * 4 + 256


def test_frequencies(W):
    f, m = W.wq_rope_frequencies(64, 10000.0)
    assert m == 1.0 and len(f) == 32 and f[0] == 1.0 and f[16] == float(torch.tensor(0.01))
    exact = [10000.0 ** (-2 * i / 64) for i in range(32)]
    near = lambda a, b: all(abs(x - y) <= 2.0 ** -24 * y * 1.01 for x, y in zip(a, b))  # noqa: E731
    assert near(f, exact)
    assert near(W.wq_rope_frequencies(64, 10000.0, W.ROPE_EVEN, 4.0)[0], [x / 4 for x in exact])
    wide = 10000.0 * 4.0 ** (64 / 62)
    assert near(W.wq_rope_frequencies(64, 10000.0, W.ROPE_BASE, 4.0)[0], [wide ** (-2 * i / 64) for i in range(32)])
    f, m = W.wq_rope_frequencies(64, 10000.0, W.ROPE_PARTS, 4.0, 4096)
    assert m == float(torch.tensor(0.1 * math.log(4.0) + 1.0))
    turns = [4096 * x / (2 * math.pi) for x in exact]
    g = [min(max((t - 1) / 31, 0.0), 1.0) for t in turns]
    assert 0.0 in g and 1.0 in g and near(f, [x * (y + (1 - y) / 4) for x, y in zip(exact, g)])
    # a factor of one changes nothing, by any rule
    for rule in (W.ROPE_EVEN, W.ROPE_BASE, W.ROPE_PARTS):
        assert W.wq_rope_frequencies(32, 500000.0, rule, 1.0, 8192) == W.wq_rope_frequencies(32, 500000.0)
    for bad in (dict(rot_dim=0, base=1e4), dict(rot_dim=-16, base=1e4), dict(rot_dim=24, base=1e4), dict(rot_dim=32, base=1.0), dict(rot_dim=32, base=math.inf),
                dict(rot_dim=32, base=1e4, scaling=4), dict(rot_dim=32, base=1e4, scaling=1, factor=0.5), dict(rot_dim=32, base=1e4, scaling=2, factor=math.nan),
                dict(rot_dim=32, base=1e4, scaling=3, factor=2.0)):
        with pytest.raises(W.WQError):
            W.wq_rope_frequencies(**bad)


def test_binding_refuses_rows_that_it_cannot_describe(W):
    """Inner strides, types and shapes that a pointer and a row stride would silently misread."""
    t = torch.zeros(4, 14, 64)
    wide = torch.zeros(4, 2000)[:, :14 * 64].unflatten(1, (14, 64))
    assert W._rows("t", t) == (4, 14, 64, 14 * 64) and W._rows("t", wide) == (4, 14, 64, 2000)
    assert W._rows("t", t[:1]) == (1, 14, 64, 14 * 64)
    with pytest.raises(ValueError):
        W._rows("t", t, t, (4, 14, 128))
    for bad in (t.transpose(0, 1), t[..., ::2], t[:, ::2], t.flatten(1)):
        with pytest.raises(ValueError):
            W._rows("t", bad)
    with pytest.raises(ValueError):
        W._rows("t", t.half(), t)
    with pytest.raises(ValueError):
        W._contiguous("off", torch.zeros(3, dtype=torch.int64), torch.int32, 3)
    with pytest.raises(ValueError):
        W._contiguous("off", torch.zeros(3, dtype=torch.int32), torch.int32, 4)
