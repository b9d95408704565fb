"""Appended rows and copied sequences at the ends of what a call may ask for."""
import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests.test_gpu_sequences import _caches

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("selected", [False, True])
def test_appending_no_row(selected):
    """max_take = 0: the caches stay as they are and no status is raised, whatever the tables hold."""
    kvs = _caches(2, 2, 2, 64, torch.bfloat16, [9, 9], [2, 0])
    x = torch.ones(6, 2, 64, dtype=torch.bfloat16, device="cuda")
    tables = (torch.empty(2, 0, dtype=torch.int32, device="cuda"), R.i32([3, -1])) if selected else (None, None)
    ctx = W.Context(0)
    W.wq_append_rows(ctx, [x, x], [x, x], kvs, R.i32([0, 3, 6]), 0, *tables)
    assert ctx.device_status() == 0
    for kv in kvs:
        assert kv.len16.tolist() == [2, 0] and bool((kv.k16 == 7).all()) and bool((kv.v16 == 9).all())


def test_layers_of_one_row_with_strides_of_their_own():
    x = torch.randn(3, 8, 2, 64, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    layers = [x[0, :1], x[1].flatten()[64:].as_strided((1, 2, 64), (1536, 64, 1)), x[2, 4:5]]
    kvs = _caches(3, 1, 2, 64, torch.bfloat16, [4], [1])
    ctx = W.Context(0)
    W.wq_append_rows(ctx, layers, layers[::-1], kvs, R.i32([0, 1]), 1)
    assert ctx.device_status() == 0
    for kv, k, v in zip(kvs, layers, layers[::-1]):
        assert kv.len16.tolist() == [2] and torch.equal(kv.k16[1], k[0]) and torch.equal(kv.v16[1], v[0])
        assert bool((kv.k16[2:] == 7).all()) and bool((kv.v16[2:] == 9).all())


def test_copied_layers_that_share_the_classes_tables():
    """Layers whose sequences have the same lengths, as one choice of bits for all of them gives."""
    lens, src = [(100, 64, 33, 20), (0, 40, 0, 3), (7, 0, 90, 0)], [2, 0, 0, 1]
    from_kv = [R.make_cache(np.random.default_rng(i), lens, 2, 64, 32, torch.bfloat16)[0] for i in range(3)]
    caps, room = [sum(-(-lens[s][c] // 32) * 32 for s in src) for c in range(3)], R.offsets([lens[s][3] for s in src])
    alone, shared = ([W.PackedKV(4, 2, 64, 32, torch.bfloat16, caps, room, fill=0) for _ in range(3)] for _ in range(2))
    for kv in shared[1:]:
        kv.cls_off, kv.cls_len = shared[0].cls_off, shared[0].cls_len
        for c in range(3):
            kv.desc.cls_off[c], kv.desc.cls_len[c] = kv.cls_off[c].data_ptr(), kv.cls_len[c].data_ptr()
    ctx = W.Context(0)
    for to in (alone, shared):
        W.wq_copy_sequences(ctx, from_kv, to, R.i32(src))
    assert ctx.device_status() == 0
    for a, b in zip(alone, shared):
        for c in range(3):
            for x, y in ((a.codes, b.codes), (a.meta, b.meta), (a.cls_off, b.cls_off), (a.cls_len, b.cls_len)):
                assert torch.equal(x[c], y[c])
        assert torch.equal(a.k16, b.k16) and torch.equal(a.v16, b.v16) and torch.equal(a.len16, b.len16) and torch.equal(a.v_scale_max[:4], b.v_scale_max[:4])
