"""Edges of the operators on the paged cache: bounds at the ends of 32 bits, plans that only large batches reach, and
streams that are not the current one.
"""
import numpy as np
import pytest
import torch

import attend_reference as ref
from harness import gpu
from paper_2609_15021_amd import attend, kvx

pytestmark = pytest.mark.gpu
DEV = ref.DEV
BF16, F16 = torch.bfloat16, torch.float16
INTS = dict(dtype=torch.int32, device=DEV)


@pytest.fixture(autouse=True)
def no_faults():
    attend.kv_attend_async_error(clear=True)
    yield
    torch.cuda.synchronize()
    assert attend.kv_attend_async_error(clear=True) == 0


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 70, 70])
@pytest.mark.parametrize("new", [[70, 3], [5, 2], [1, 1]])
def test_windows_that_hide_nothing(window, new):
    """The widest windows are no window, for rows that would lie before token 0 too: outputs and received weights."""
    c = ref.Case(2, 3, 64, 16, [3, 40], new, seed=31)
    cache, _, q, _, _, tables, lens, starts = c.device()
    want = ref.attend(c)
    weights = torch.zeros(2, 2, 40, device=DEV)
    out, lse = attend.kv_attend(cache, 0, q, tables, lens, starts, window=window, weights=weights)
    ref.check(out, want[0], want[3], "out")
    ref.check(lse, want[1], want[4], "lse")
    for b, n in enumerate(c.lens):
        ref.check(weights[b, :, :n], want[2][b, :, :n], want[5][b, :, :n], "weights")
