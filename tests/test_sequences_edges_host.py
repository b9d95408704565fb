"""Calls for appended rows and copied sequences that the caller may make and that refusals could hit, or miss (no GPU is needed)."""
import pytest
import torch

from tests.test_operators_host import W, _desc, ctx  # noqa: F401  (fixtures)
from tests.test_tree_host import _append, _other


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
