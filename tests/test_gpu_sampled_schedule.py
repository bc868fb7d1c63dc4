"""The serving schedules with drawn tokens: at temperature 0 they are the greedy ones, and
otherwise every step's picks are the definition's for its logits and its u."""

import numpy as np
import pytest
import torch

import workloads as W
from paper_2608_26140_amd import driver as D
from paper_2608_26140_amd import workload as WL
from tests import paged_reference as R
from tests.gpu_util import up
from tests.oracle_side import anchor_count

pytestmark = pytest.mark.gpu


def setup():
    w = W.get_config("mini-serve")
    s = WL.build(w)
    g, h = W.draw_lm_head(w)
    K, blk = anchor_count(w), w.decode_block
    plan = D.DecodePlan(s.batch, K, blk, w.layout.mask_len // blk, full=False)
    return w, s.batch, D.Head(up(g, w.dims.dtype), up(h, w.dims.dtype)), plan, K, blk


def seeded(n):
    return torch.Generator(device="cuda").manual_seed(n)


def test_schedule_at_temperature_0_is_greedy():
    w, batch, head, plan, K, blk = setup()
    ids = batch.remap.clone()
    anchors, _ = batch.select_anchors(K)
    logits = torch.empty((batch.B * blk, w.dims.vocab), dtype=torch.bfloat16, device="cuda")
    res = []
    for sampling in (None, D.Sampling(batch, blk, temperature=0.0), D.Sampling(batch, blk, temperature=[0.0] * batch.B, top_k=7)):
        batch.remap.copy_(ids)
        out = torch.full((plan.n_blocks, batch.B * blk), -1, dtype=torch.int32, device="cuda")
        D.decode_schedule(batch, head, plan, K, logits, out, anchors=anchors, sampling=sampling)
        res.append((out, batch.remap.clone()))
    for out, after in res[1:]:
        assert torch.equal(out, res[0][0]) and torch.equal(after, res[0][1])


def test_threshold_schedule_draws_by_the_definition():
    w, batch, head, plan, K, blk = setup()
    ids = batch.remap.clone()
    anchors, _ = batch.select_anchors(K)
    per = dict(temperature=[0.6, 1.0, 0.0], top_k=[40, 0, 3], top_p=[0.9, 1.0, 0.5], min_p=[0.0, 0.01, 0.0])
    assert batch.B == 3
    runs = []
    for _ in range(2):  # the same seed, the same tokens
        batch.remap.copy_(ids)
        trace = []
        D.decode_threshold_schedule(batch, head, plan, K, 0.004, anchors=anchors, trace=trace, max_steps=3,
                                    sampling=D.Sampling(batch, blk, **per, generator=seeded(7)))
        runs.append((trace, batch.remap.clone()))
    assert torch.equal(runs[0][1], runs[1][1])
    gen, u = seeded(7), torch.empty(batch.B * blk, dtype=torch.float64, device="cuda")
    rows = {n: np.repeat(np.asarray(v, dtype=np.float32), blk) for n, v in per.items()}
    assert len(runs[0][0]) >= plan.n_blocks
    for a, b in zip(*[r[0] for r in runs]):
        assert np.array_equal(a["pick"], b["pick"])
        u.uniform_(generator=gen)
        want, conf, _ = R.sample(a["logits"], u.cpu().numpy(), **rows, got=a["pick"])
        assert np.array_equal(a["pick"], want)
        assert np.all(np.abs(a["conf"] - conf) <= 2.0 ** -23 * conf)


def test_settings_that_do_not_fit_are_refused():
    w, batch, *_, blk = setup()
    with pytest.raises(ValueError):
        D.Sampling(batch, blk, temperature=[1.0] * (batch.B + 1))
    with pytest.raises(ValueError):
        D.Sampling(batch, blk, top_p=[[1.0] * batch.B])
