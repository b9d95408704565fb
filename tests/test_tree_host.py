"""Refusals of the calls for several new rows per sequence and for copies of sequences: reported before anything is enqueued, so no GPU is needed."""
import ctypes as C
import math

import pytest
import torch

from tests.test_operators_host import P, W, _desc, ctx  # noqa: F401  (fixtures)

BF, F16, F32 = 1, 2, 0


def _tree(W, ctx, d=None, **more):
    a = dict(q=P, qs=14 * 64, k=P, ks=128, v=P, vs=128, dtype=BF, B=2, Hq=14, ro=P, par=P, rows=100, mr=50, sm=0.125, splits=1, mc=1000, out=P, lse=None)
    a.update(more)
    return W.lib().wq_tree_attention(ctx, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], a["B"], a["Hq"], C.byref(d or _desc(W)), a["ro"], a["par"],
                                     a["rows"], a["mr"], a["sm"], a["splits"], a["mc"], a["out"], a["lse"])


@pytest.mark.parametrize("bad,code", [
    (dict(B=-1), -1), (dict(B=3), -1), (dict(rows=-1), -1), (dict(mr=-1), -1), (dict(mc=-1), -1), (dict(dtype=3), -1), (dict(dtype=F16), -1), (dict(dtype=F32), -1),
    (dict(Hq=15), -2), (dict(Hq=18, qs=18 * 64), -2), (dict(Hq=0), -2), (dict(rows=1 << 31), -2), (dict(mr=1025), -2), (dict(splits=-1), -1), (dict(splits=65), -1),
    (dict(sm=0.0), -1), (dict(sm=-1.0), -1), (dict(sm=math.nan), -1), (dict(sm=math.inf), -1), (dict(sm=3e38), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1),
    (dict(ro=None), -1), (dict(out=None), -1), (dict(out=P + 8), -1), (dict(q=P + 8), -1), (dict(k=P + 2), -1), (dict(qs=100), -1), (dict(ks=132), -1), (dict(vs=64), -1),
    (dict(ks=(1 << 22) + 8), -2), (dict(vs=1 << 23), -2), (dict(splits=64), -4), (dict(rows=100000, splits=2, mr=0), -4)])
def test_tree_attention_refuses(W, ctx, bad, code):  # noqa: F811
    assert _tree(W, ctx, **bad) == code
    assert W.lib().wq_last_error(ctx)


def test_tree_attention_refuses_caches(W, ctx):  # noqa: F811
    assert W.lib().wq_tree_attention(ctx, P, 896, P, 128, P, 128, BF, 2, 14, None, P, P, 10, 5, 0.125, 1, 10, P, None) == -1
    for more, code in ((dict(hd=96), -2), (dict(group=128), -2), (dict(dtype16=F16), -1), (dict(Hkv=4), -2)):
        assert _tree(W, ctx, _desc(W, **more)) == code
    for name in ("k16", "v16"):
        d = _desc(W)
        setattr(d, name, P + 8)
        assert _tree(W, ctx, d) == -1
    d = _desc(W)
    d.codes[1] = P + 4
    assert _tree(W, ctx, d) == -1
    d = _desc(W)
    d.cls_len[2] = None
    assert _tree(W, ctx, d) == -1
    wide = _desc(W, Hkv=1 << 17)
    assert _tree(W, ctx, wide, Hq=1 << 19, qs=1 << 25, ks=1 << 23, vs=1 << 23) == -2


def test_tree_attention_without_rows(W, ctx):  # noqa: F811
    assert _tree(W, ctx, rows=0) == 0 and _tree(W, ctx, rows=0, q=None, k=None, v=None, ro=None, out=None) == 0
    assert _tree(W, ctx, _desc(W, B=0), B=0) == 0
    assert W.lib().wq_tree_attention(None, *([None, 0] * 3), 0, 0, 1, None, None, None, 0, 0, 1.0, 0, 0, None, None) == -1
    # parts that the join's grid cannot hold: refused if asked for, else fewer
    many = dict(B=65535, Hq=64, rows=65535 * 12, qs=64 * 64, ks=8 * 64, vs=8 * 64, mr=17, par=None)
    assert _tree(W, ctx, _desc(W, Hkv=8, B=65535), splits=2, **many) == -2
    assert W.tree_workspace_bytes(65535 * 12, 65535, 64, 8, 64, 1 << 62, (1 << 31) - 1) == 16384
    # a chain has no bound of 1024 rows; a workspace without room for parts is enough for one
    assert _tree(W, ctx, par=None, mr=2000, rows=4000, splits=64) == -4


def test_tree_workspace_bytes(W):  # noqa: F811
    f = W.tree_workspace_bytes
    assert f(0, 1, 14, 2, 64, 1000, 10) == f(10, 0, 14, 2, 64, 1000, 10) == f(10, 1, 15, 2, 64, 1000, 10) == 16384
    assert f(10, 1, 14, 2, 64, 1000, 10, 1) == 16384 and f(10, (1 << 31) - 1, 14, 2, 64, (1 << 63) - 1, 10, 1) == 16384
    assert f(10, 1, 14, 2, 64, 1000, 10, 4) >= 16384 + 10 * 14 * 4 * 66 * 4
    assert f(10, 1, 14, 2, 64, 10 ** 6, 10) > f(10, 1, 14, 2, 64, 1000, 10, 1)


def _accept(W, ctx, **more):
    a = dict(tok=P, tgt=P, par=P, B=2, ro=P, rows=10, mr=8, mp=4, path=P, n=P, nxt=P)
    a.update(more)
    return W.lib().wq_tree_accept(ctx, a["tok"], a["tgt"], a["par"], a["B"], a["ro"], a["rows"], a["mr"], a["mp"], a["path"], a["n"], a["nxt"])


@pytest.mark.parametrize("bad,code", [
    (dict(B=-1), -1), (dict(rows=-1), -1), (dict(mr=0), -1), (dict(mp=0), -1), (dict(mr=1025), -2), (dict(B=1 << 24), -2), (dict(tok=None), -1), (dict(tgt=None), -1),
    (dict(ro=None), -1), (dict(path=None), -1), (dict(n=None), -1), (dict(nxt=None), -1)])
def test_accept_refuses(W, ctx, bad, code):  # noqa: F811
    assert _accept(W, ctx, **bad) == code
    assert W.lib().wq_last_error(ctx)
    assert _accept(W, ctx, B=0, ro=None) == 0 and _accept(W, None) == -1


def _append(W, ctx, ds=None, k=(P, P), v=(P, P), **more):
    a = dict(n=2, ks=128, vs=128, dtype=BF, B=2, ro=P, rows=10, take=P, nt=P, mt=4)
    a.update(more)
    ds = ds or [_desc(W), _other(W)]
    arr = C.c_void_p * 2
    return W.lib().wq_append_rows(ctx, a["n"], None if k is None else arr(*k), a["ks"], None if v is None else arr(*v), a["vs"], a["dtype"], a["B"], a["ro"], a["rows"],
                                  a["take"], a["nt"], a["mt"], (W._PackedKV * 2)(*ds))


@pytest.mark.parametrize("bad,code", [
    (dict(n=-1), -1), (dict(B=-1), -1), (dict(B=3), -1), (dict(rows=-1), -1), (dict(mt=-1), -1), (dict(dtype=5), -1), (dict(dtype=F32), -1), (dict(take=None), -1), (dict(nt=None), -1),
    (dict(ro=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(k=(P, None)), -1), (dict(v=(P + 8, P)), -1), (dict(ks=64), -1), (dict(vs=130), -1)])
def test_append_rows_refuses(W, ctx, bad, code):  # noqa: F811
    assert _append(W, ctx, **bad) == code
    assert W.lib().wq_last_error(ctx)


def test_append_rows_refuses_caches(W, ctx):  # noqa: F811
    for more in (dict(Hkv=4), dict(hd=128), dict(dtype16=F16)):
        assert _append(W, ctx, [_desc(W), _other(W, **more)]) == -1
    d = _desc(W)
    d.v16 = P + 8
    assert _append(W, ctx, [_desc(W), d]) == -1
    d = _desc(W)
    d.len16 = None
    assert _append(W, ctx, [d, _desc(W)]) == -1
    assert _append(W, ctx, [_desc(W, B=1 << 20), _other(W, B=1 << 20)], B=1 << 20, mt=1 << 20, take=None, nt=None) == -2
    assert _append(W, ctx, mt=(1 << 31) - 1, take=None, nt=None) == -2       # (rounded up in 32 bits it would be negative)
    assert _append(W, ctx, [_desc(W), _desc(W)]) == -1                       # the same cache twice
    d = _other(W)
    d.len16 = P
    assert _append(W, ctx, [_desc(W), d]) == -1
    assert _append(W, ctx, n=0) == 0 and _append(W, ctx, rows=0, k=(None, None), v=(None, None), take=None, nt=None) == 0 and _append(W, ctx, mt=0) == 0
    assert _append(W, None) == -1


def _copy(W, ctx, src, dst, n=1, frm=P):
    return W.lib().wq_copy_sequences(ctx, n, (W._PackedKV * len(src))(*src), (W._PackedKV * len(dst))(*dst), frm)


def _other(W, at=0x100000, **more):
    d = _desc(W, **more)
    for c in range(3):
        d.codes[c], d.meta[c], d.cls_off[c], d.cls_len[c] = at, at, at, at
    d.k16 = d.v16 = d.off16 = d.len16 = d.v_scale_max = at
    return d


def test_copy_refuses(W, ctx):  # noqa: F811
    lib = W.lib()
    assert _copy(W, ctx, [_desc(W)], [_other(W)], n=-1) == -1 and _copy(W, ctx, [_desc(W)], [_other(W)], frm=None) == -1
    assert lib.wq_copy_sequences(ctx, 1, None, C.byref(_desc(W)), P) == -1 and lib.wq_copy_sequences(ctx, 1, C.byref(_desc(W)), None, P) == -1
    for more, code in ((dict(Hkv=4), -1), (dict(hd=128), -1), (dict(group=64), -1), (dict(dtype16=F16), -1), (dict(hd=96), -2), (dict(B=65536), -2)):
        assert _copy(W, ctx, [_desc(W)], [_other(W, **more)]) == code
        assert lib.wq_last_error(ctx)
    assert _copy(W, ctx, [_desc(W)], [_desc(W)]) == -1                       # onto itself
    for name in ("k16", "v16", "len16", "v_scale_max"):
        d = _other(W)
        setattr(d, name, P)
        assert _copy(W, ctx, [_desc(W)], [d]) == -1
    for name in ("codes", "meta", "cls_off", "cls_len"):
        d = _other(W)
        getattr(d, name)[1] = P
        assert _copy(W, ctx, [_desc(W)], [d]) == -1
    d = _other(W)
    d.codes[0] = 0x100008
    assert _copy(W, ctx, [_desc(W)], [d]) == -1
    assert _copy(W, ctx, [_desc(W), _desc(W, B=3)], [_other(W), _other(W)], n=2) == -1
    assert _copy(W, ctx, [_desc(W)], [_other(W, B=0)]) == 0 and _copy(W, ctx, [_desc(W)], [_other(W)], n=0) == 0 and _copy(W, None, [_desc(W)], [_other(W)]) == -1


def test_python_calls_refuse(W):  # noqa: F811
    """What the binding checks itself: shapes, types, tables, devices."""
    class Cpu:                                                               # a context whose device is the host
        index, device, handle = -1, torch.device("cpu"), None

        def check(self, rc):
            raise AssertionError("reached the library")
    kv = W.PackedKV(2, 2, 64, 32, torch.bfloat16, [0, 0, 0], [0, 8, 16], device="cpu")
    q, k, off = torch.zeros(5, 14, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    ok = dict(q=q, k=k, v=k, kv=kv, row_off=off, sm_scale=0.1)
    for bad in (dict(q=q[..., :32]), dict(k=k[:4]), dict(v=k.float()), dict(k=k[:, :1]), dict(row_off=off[:2]), dict(row_off=off.long()), dict(parent=off),
                dict(parent=torch.zeros(5)), dict(out=q.float()), dict(lse=torch.zeros(5, 13)), dict(q=q.transpose(0, 1))):
        with pytest.raises(ValueError):
            W.wq_tree_attention(Cpu(), **{**ok, **bad})
    tok = torch.zeros(5, dtype=torch.int32)
    for bad in (dict(target=tok[:4]), dict(tokens=tok.long(), target=tok), dict(row_off=off.long()), dict(parent=tok[:3])):
        with pytest.raises(ValueError):
            W.wq_tree_accept(Cpu(), **{**dict(tokens=tok, target=tok, row_off=off), **bad})
    rows = dict(k=[k, k], v=[k, k], kv=[kv, kv], row_off=off, max_take=3)
    for bad in (dict(k=[k]), dict(kv=[]), dict(k=[k, k.float()], v=[k, k]), dict(k=[k, k[:4]]), dict(v=[k, k.float()]), dict(k=[k, torch.zeros(5, 3, 64, dtype=torch.bfloat16)[:, :2]]), dict(row_off=off[:2]),
                dict(take=torch.zeros(2, 3, dtype=torch.int32)), dict(take=torch.zeros(2, 2, dtype=torch.int32), n_take=off[:2]), dict(k=[k[:, :1]] * 2, v=[k[:, :1]] * 2)):
        with pytest.raises(ValueError):
            W.wq_append_rows(Cpu(), **{**rows, **bad})
    for bad in (([kv], [kv, kv], off), ([], [], off), ([kv], [kv], off), ([kv], [kv], off[:2].long())):
        with pytest.raises(ValueError):
            W.wq_copy_sequences(Cpu(), *bad)
