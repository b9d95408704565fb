"""Calls for appended rows and copied sequences that the caller may make and that refusals could hit, or miss (no GPU is needed)."""
import pytest
import torch

from tests.test_operators_host import W, _desc, ctx  # noqa: F401  (fixtures)
from tests.test_tree_host import _append, _copy, _other


@pytest.mark.parametrize("tables", [dict(), dict(take=None), dict(take=None, nt=None), dict(nt=None)])
def test_no_row_may_be_appended(W, ctx, tables):  # noqa: F811
    """With max_take = 0 a table of rows has no columns, and an empty tensor no address."""
    assert _append(W, ctx, mt=0, **tables) == 0


@pytest.mark.parametrize("mine,other", [("k16", "k16"), ("k16", "v16"), ("v16", "k16"), ("v16", "v16"), ("len16", "len16")])
def test_layers_that_share_rows(W, ctx, mine, other):  # noqa: F811
    """Two layers' workgroups would write the same rows."""
    a, b = _desc(W), _other(W)
    a.v16, b.v16 = 0x2000, 0x200000
    assert _append(W, ctx, [a, b], mt=0) == 0
    setattr(b, other, getattr(a, mine))
    assert _append(W, ctx, [a, b], mt=0) == -1 and W.lib().wq_last_error(ctx)
    assert _append(W, ctx, [b, a], mt=0) == -1


def test_layers_without_rows_share_nothing(W, ctx):  # noqa: F811
    """Buffers of no rows may have any address."""
    a, b = _desc(W, cap16=0), _other(W, cap16=0)
    b.k16 = b.v16 = a.k16
    assert _append(W, ctx, [a, b], mt=0) == 0


def _apart(W, at, layer):  # noqa: F811
    """A cache whose buffers and tables all have addresses of their own."""
    d, n = _other(W), [at + layer * 0x100000]

    def new():
        n[0] += 0x1000
        return n[0]
    for c in range(3):
        d.codes[c], d.meta[c], d.cls_off[c], d.cls_len[c] = new(), new(), new(), new()
    d.k16, d.v16, d.off16, d.len16, d.v_scale_max = new(), new(), new(), new(), new()
    return d


BUFFERS = ["codes", "meta", "cls_off", "cls_len", "k16", "v16", "len16", "v_scale_max"]
TABLES = BUFFERS[2:4]


def _get(d, name):
    return getattr(d, name)[1] if name in BUFFERS[:4] else getattr(d, name)


def _set(d, name, value):
    if name in BUFFERS[:4]:
        getattr(d, name)[1] = value
    else:
        setattr(d, name, value)


@pytest.mark.parametrize("mine", BUFFERS)
@pytest.mark.parametrize("other", BUFFERS)
def test_copies_that_share_memory(W, ctx, mine, other):  # noqa: F811
    """A buffer of one layer's copy that is also another layer's, or a source's, would be written by both, or while it is read."""
    src, dst = ([_apart(W, at, i) for i in range(3)] for at in (0x10000000, 0x20000000))
    for d in src + dst:
        d.B = 2
    def call():
        code = _copy(W, ctx, src, dst, n=3, frm=None)                    # (refused in the end: no table of sources)
        return code, W.lib().wq_last_error(ctx)
    assert call() == (-1, b"from is NULL")
    for a, b in ((dst[0], dst[2]), (dst[2], dst[0]), (src[0], dst[2]), (src[1], dst[0]), (src[2], dst[2])):
        kept = _get(b, other)
        _set(b, other, _get(a, mine))
        code, why = call()
        if a in dst and mine in TABLES and other in TABLES:              # (tables that are written alike)
            assert why == b"from is NULL"
        else:
            assert code == -1 and b"memory" in why, (mine, other)
        _set(b, other, kept)
    assert call() == (-1, b"from is NULL")


def test_copies_may_share_what_they_read_or_write_alike(W, ctx):  # noqa: F811
    src, dst = ([_apart(W, at, i) for i in range(3)] for at in (0x10000000, 0x20000000))
    dst[0].off16 = dst[1].off16 = src[0].off16 = src[2].off16            # where the 16-bit segments lie
    src[1] = src[0]                                                      # one source for two layers
    for c in range(3):                                                   # layers of the same lengths
        dst[1].cls_off[c], dst[1].cls_len[c] = dst[0].cls_off[c], dst[0].cls_len[c]
    for d in dst:                                                        # buffers of no tokens
        d.cap[0] = d.cap16 = 0
        d.codes[0], d.meta[0], d.k16, d.v16 = src[0].codes[0], src[0].meta[0], src[0].k16, src[0].v16
    assert _copy(W, ctx, src, dst, n=3, frm=None) == -1 and W.lib().wq_last_error(ctx) == b"from is NULL"
    many = [_apart(W, 0x100000000, i) for i in range(700)]               # (more addresses than a filter tells apart)
    to = [_apart(W, 0x200000000, i) for i in range(700)]
    arr = W._PackedKV * 700
    assert W.lib().wq_copy_sequences(ctx, 700, arr(*many), arr(*to), None) == -1 and W.lib().wq_last_error(ctx) == b"from is NULL"
    to[699].meta[2] = to[3].k16
    assert W.lib().wq_copy_sequences(ctx, 700, arr(*many), arr(*to), None) == -1 and b"memory" in W.lib().wq_last_error(ctx)


class _Cpu:
    """A context whose device is the host: a call that the binding lets through ends here."""
    index, device, handle = -1, torch.device("cpu"), None

    def check(self, rc):
        raise KeyError("reached the library")


def _rows(rows, heads, *strides):
    """The same rows in layers with these strides."""
    return [torch.zeros(4096, dtype=torch.bfloat16).as_strided((rows, heads, 64), s) for s in strides]


def _append_layers(W, k, v):  # noqa: F811
    heads = k[0].shape[1]
    kvs = [W.PackedKV(2, heads, 64, 32, torch.bfloat16, [0, 0, 0], [0, 8, 16], device="cpu") for _ in k]
    W.wq_append_rows(_Cpu(), k, v, kvs, torch.zeros(3, dtype=torch.int32), 3)


def test_strides_that_say_nothing(W):  # noqa: F811
    """One row, or one head: how far the next would be away differs from layer to layer, and no next one is read."""
    for k in (_rows(1, 2, (128, 64, 1), (1536, 64, 1), (64, 64, 1)), _rows(5, 1, (128, 64, 1), (128, 128, 1), (128, 7, 1)), _rows(1, 1, (64, 64, 1), (1, 3, 1), (72, 64, 1)),
              _rows(0, 2, (128, 64, 1), (256, 64, 1), (0, 0, 1))):
        for a, b in ((k, k), (k, [k[0]] * 3), ([k[1]] * 3, k)):
            with pytest.raises(KeyError):
                _append_layers(W, a, b)


def test_strides_that_differ(W):  # noqa: F811
    plain = _rows(2, 2, (128, 64, 1)) * 2
    for k in (_rows(2, 2, (128, 64, 1), (192, 64, 1)), _rows(2, 1, (128, 64, 1), (192, 64, 1)), _rows(1, 2, (128, 64, 1), (128, 128, 1)), _rows(2, 2, (128, 64, 1), (64, 128, 1)),
              _rows(2, 2, (128, 64, 1), (256, 64, 2))):
        same = plain if k[0].shape == plain[0].shape else [k[0], k[0]]
        for a, b in ((k, same), (same, k)):
            with pytest.raises(ValueError):
                _append_layers(W, a, b)
