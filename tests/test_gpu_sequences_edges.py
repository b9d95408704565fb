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
