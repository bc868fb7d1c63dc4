"""Stores into the 8-bit cache whose workspace holds what earlier calls, or
nothing, left there: the result is the definition's whatever the contents."""

import numpy as np
import pytest
import torch

from tests.test_gpu_quant import Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("past", [0, 1, 43])
def test_store_after_a_store_whose_last_row_is_now_past_the_end(past):
    """The first call leaves its last row as the short last block's.  The second
    stores that block in its first rows, and in that last row names no slot, by
    a number in the block's range."""
    n_slots, n = 32 * 64 + 20, 1500
    p = Pair("bf16", 2, 128, n_slots, 64, seed=past)
    p.store(np.arange(n_slots - n, n_slots))
    slots = np.concatenate([np.arange(n_slots - 20, n_slots), np.arange(n - 21), [n_slots + past]])
    p.store(slots, 3.0)
    p.store(np.concatenate([slots[20:-1], slots[:20], [n_slots + past]]), 0.5)  # the block's rows next to it


@pytest.mark.parametrize("row", [0, 5, 19, 20, 700, 1400, 1480, 1498, 1499, 1500, -1])
@pytest.mark.parametrize("block", [16, 64, 256])
def test_store_into_any_workspace(row, block):
    """Every entry of the workspace holds the number of one row: of one in the
    last block, elsewhere, without a slot, or of none."""
    n_slots, n = 8 * 256 + 13, 1500
    p = Pair("bf16", 1, 128, n_slots, block, seed=block)
    p.ws.view(torch.int32).fill_(row)
    slots = np.concatenate([np.arange(n_slots - 20, n_slots), np.arange(n - 40), n_slots + np.arange(20) % 3])
    p.store(slots)
    p.ws.view(torch.int32).fill_(row)
    p.store(slots[::-1].copy(), 4.0)
