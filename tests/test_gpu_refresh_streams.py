"""The baselines' refreshes on a stream of their own: the same rows as on the
current one, behind what that stream still does."""

import pytest
import torch

import workloads as W
from paper_2608_26140_amd import workload as WL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["direct_reuse", "full_refresh"])
@pytest.mark.parametrize("name", ["mini-stack", "mini-f32-stack"])
def test_baseline_refresh_on_another_stream(name, call):
    batch = WL.build(W.get_config(name), keep_host=False).batch
    want = getattr(batch, call)()[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    rows = batch.x_src.clone()
    batch.x_src.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        batch.x_src.copy_(rows)
    got, _ = getattr(batch, call)(stream=side)
    side.synchronize()
    assert torch.equal(got, want)
