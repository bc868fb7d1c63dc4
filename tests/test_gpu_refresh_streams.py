"""The baselines' refreshes on a stream of their own: the same rows as on the
current one, behind what that stream still does."""

import pytest
import torch

import workloads as W
from paper_2608_26140_amd import acache as A
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


@pytest.mark.parametrize("name,qb", [("mini-stack", None), ("mini-stack", 64), ("mini-f32-stack", None)])
def test_calls_on_another_stream_do_not_wait_for_the_current_one(name, qb):
    """What a call makes for itself (an index of every affix row, scores, maps)
    is made on its stream, also while the current stream is busy; memory that it
    frees is not the current stream's to take."""
    w = W.get_config(name)
    batch = WL.build(w, keep_host=False, quant_block=qb).batch
    k = A.acache_anchor_count(w.ratio, batch.L)

    def run(stream=None):
        anchors, scores = batch.select_anchors(k, stream=stream)
        out = [anchors, scores, batch.refresh(anchors, k, stream=stream)[0], batch.full_refresh(stream)[0]]
        if not qb:
            out += batch.select_anchors_hkvd(k, stream=stream)
        return out
    want = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    got = run(side)
    scrap = [torch.full((w.batch * batch.S * w.dims.d_model,), 7.0, device="cuda", dtype=batch.model.dtype)
             for _ in range(4)]
    side.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), f"output {i}"
    assert all((t == 7).all() for t in scrap)
