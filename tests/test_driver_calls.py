"""What the driver's baselines pass on to the refresh.  CPU only."""

import pytest
import torch

from paper_2608_26140_amd.driver import AffixBatch


@pytest.mark.parametrize("call,k", [("direct_reuse", 0), ("full_refresh", 5)])
def test_baselines_pass_their_stream_as_a_stream(call, k):
    batch = AffixBatch.__new__(AffixBatch)
    batch.L, batch.B, batch.device = 5, 2, "cpu"
    seen = {}

    def refresh(anchors, k, drop_non_anchor=False, stream=None, layer_hook=None):
        seen.update(anchors=anchors, k=k, drop=drop_non_anchor, stream=stream)
    batch.refresh = refresh
    stream = object()
    getattr(batch, call)(stream)
    assert seen["k"] == k and seen["drop"] is False and seen["stream"] is stream
    if k:
        assert torch.equal(seen["anchors"], torch.arange(5, dtype=torch.int32).repeat(2, 1))
