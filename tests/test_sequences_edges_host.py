"""Calls for appended rows and copied sequences that the caller may make and that refusals could hit, or miss (no GPU is needed)."""
import pytest
import torch

from tests.test_operators_host import W, _desc, ctx  # noqa: F401  (fixtures)
from tests.test_tree_host import _append


@pytest.mark.parametrize("tables", [dict(), dict(take=None), dict(take=None, nt=None), dict(nt=None)])
def test_no_row_may_be_appended(W, ctx, tables):  # noqa: F811
    """With max_take = 0 a table of rows has no columns, and an empty tensor no address."""
    assert _append(W, ctx, mt=0, **tables) == 0
