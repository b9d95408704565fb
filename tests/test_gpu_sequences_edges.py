"""Appended rows and copied sequences at the ends of what a call may ask for."""
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
