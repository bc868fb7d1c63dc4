"""Emptying blocks of an 8-bit cache on a stream of its own."""

import pytest
import torch

from paper_2608_26140_amd import acache as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slots,left", [(None, [0, 0, 0, 0]), (slice(10, 50), [1, 0, 0, 1])])
def test_clear_on_another_stream(slots, left):
    """Behind what that stream still does, in order with its other calls."""
    pool = A.quant_pool(A.make_dims(256, 2, 2, 128, 256, "bf16"), 60, 16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        pool.k_scales.fill_(1.0)
        pool.v_scales.fill_(1.0)
    pool.clear(slots, stream=side)
    side.synchronize()
    for t in (pool.k_scales, pool.v_scales):
        assert t[:, 0].tolist() == left and t[:, 1].tolist() == left
