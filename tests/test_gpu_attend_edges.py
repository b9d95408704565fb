"""Prompt attention and shared decode where a call is out of the ordinary: a workspace that was sized for another call, queries of zero and scales at the
ends of fp32, NaN, values far beyond fp16, and how much of a 16-bit call's accuracy its roundings take."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import test_gpu_prefill as P
from tests import test_gpu_shared_prefix as S

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
SMALL, LARGE = (14, 2, 64), (28, 4, 128)


# ---- a workspace that was sized for another call ---------------------------------------------------------------------
@pytest.mark.parametrize("new,rows,prefix,heads,largest", [
    ([400], [6400], [0], LARGE, (6400, 6400)),                     # parts, where the largest call has none
    ([1, 1, 1], [900, 6400, 77], None, SMALL, (8000, 6400)),       # ... of single tokens
    ([4400], [4400], [4400], (16, 16, 64), (6400, 6400)),          # a cut last round, where the largest call has none
    ([4400], [4400], [4400], (16, 16, 64), None),                  # room for some of its parts
    ([40], [3000], None, LARGE, None)])
def test_prompts_on_a_workspace_for_a_larger_call(monkeypatch, new, rows, prefix, heads, largest):
    ample = W.prefill_workspace_bytes(sum(new), len(new), *heads, max(rows))
    size = W.prefill_workspace_bytes(largest[0], 1, *heads, largest[1]) if largest else 16384 + (ample - 16384) // 2
    assert 16384 <= size < ample
    monkeypatch.setattr(W, "prefill_workspace_bytes", lambda *a: size)
    P._check(new, rows, prefix, *heads, torch.bfloat16, 0, every=37 if sum(new) > 1000 else 7)


@pytest.mark.parametrize("B,largest,own", [(32, 37, None), (32, 37, (0, 0, 0, 9)), (31, 39, (40, 0, 9, 11)), (30, 37, (0, 0, 0, 1500))])
@pytest.mark.parametrize("dtype", DTYPES[1:])
def test_shared_caches_on_a_workspace_for_a_larger_call(monkeypatch, B, largest, own, dtype):
    longest, longest_own = (2100, sum(own) if own else 0)
    size = W.shared_workspace_bytes(largest, 1, *SMALL, longest, longest_own)
    assert size < W.shared_workspace_bytes(B, 1, *SMALL, longest, longest_own)
    # (and one that holds a single part of everything, the least that any call of this size has been sized for)
    for bytes_ in (size, W.shared_workspace_bytes(B, 1, *SMALL, 1, 1, 1)):
        with monkeypatch.context() as m:
            m.setattr(W, "shared_workspace_bytes", lambda *a: bytes_)
            S._check([(700, 900, 400, 100)], [B], None if own is None else [own] * B, SMALL, 32, dtype)
