"""Slots of 8-bit caches that served something else before: a batch whose
blocks carry an earlier occupant's scales gives the bits of a fresh batch.

The earlier occupant's rows are about 2^8 times the ones to come and fill every
slot outside the affix (or every slot), so a scale that outlived it would round
everything stored beside it to zero."""

import numpy as np
import pytest
import torch

import workloads as W
from paper_2608_26140_amd import acache as A
from paper_2608_26140_amd import driver as D
from paper_2608_26140_amd import workload as WL
from tests.gpu_util import up_i32
from tests.oracle_side import anchor_count

pytestmark = pytest.mark.gpu

PLANS = [("mini-stack", 64, None), ("mini-stack", 32, 64), ("mini-affix64", 32, 64), ("mini-affix64", 128, None),
         ("mini-gqa-infix", 64, 128)]


def occupy(batch, slots):
    """Large rows in the given slots of every layer."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x = (300 * torch.randn(len(slots), batch.model.kv_width, generator=g, device="cuda")).to(torch.bfloat16)
    for c in batch.caches:
        A.acache_quant_store(batch.model.dims, c, x, x.flip(0).contiguous(), up_i32(slots))


def private(batch):
    """Every slot that a request can be given.  (Those between the affix's last
    slot and the end of its block are given to none: they share its scale.)"""
    return np.arange(batch.first_private * batch.quant_block, batch.n_slots)


def chain(batch, w):
    """Probe, selection, refresh and two decode steps; what they leave in the
    request's slots too."""
    k = anchor_count(w)
    anchors, scores = batch.select_anchors(k)
    x, m = batch.refresh(anchors, k)
    x = x.clone()
    out = [anchors, scores, x]
    for c in batch.caches:
        out += A.acache_quant_load(batch.model.dims, c, m["write_slots"])
        out += [s[m["write_slots"].long() // batch.quant_block] for s in (c.k_scales, c.v_scales)]
    blen = 8
    plan = D.DecodePlan(batch, k, blen, w.layout.mask_len // blen, full=False)
    for blk in (0, 1):
        out.append(D.decode_step(batch, plan, blk, m, anchors))
    return out


def equal(got, want):
    assert len(got) == len(want)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), f"output {i}"


@pytest.mark.parametrize("name,qb,paged", PLANS)
def test_earlier_private_rows_leave_nothing(name, qb, paged):
    w = W.get_config(name)
    fresh, used = (WL.build(w, quant_block=qb, block_size=paged).batch for _ in range(2))
    occupy(used, private(used))
    want = chain(fresh, w)
    equal(chain(used, w), want)
    occupy(used, private(used))  # between two prompts, the table of the first still held
    equal(chain(used, w), want)
    if paged:
        used.release_private()
        occupy(used, private(used))
        equal(chain(used, w), want)
    equal(chain(fresh, w), want)  # and after itself


@pytest.mark.parametrize("name,qb,paged", PLANS[:3])
def test_full_and_direct_refreshes(name, qb, paged):
    """Every row, and no anchor: the table grows and shrinks between them."""
    w = W.get_config(name)
    fresh, used = (WL.build(w, quant_block=qb, block_size=paged).batch for _ in range(2))
    want = [t.clone() for t in (fresh.direct_reuse()[0], fresh.full_refresh()[0], fresh.direct_reuse()[0])]
    assert torch.equal(want[0], want[2])
    occupy(used, private(used))
    for i, call in enumerate((used.direct_reuse, used.full_refresh, used.direct_reuse)):
        assert torch.equal(call()[0], want[i]), i


def test_another_stream():
    """The blocks are emptied on the call's stream, behind what it still does."""
    w = W.get_config("mini-stack")
    fresh, used = (WL.build(w, quant_block=64).batch for _ in range(2))
    want, _ = fresh.direct_reuse()
    slots, side = private(used), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        occupy(used, slots)
    got, _ = used.direct_reuse(stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_captured_without_a_run_before():
    """The first eager chain, replays and eager chains give the same bits."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64, keep_host=False).batch

    def run():
        k = anchor_count(w)
        anchors, scores = batch.select_anchors(k)
        return anchors, scores, batch.refresh(anchors, k)[0]
    want = [t.clone() for t in run()]
    graph, out = D.capture(run)
    slots = private(batch)
    for _ in range(3):
        occupy(batch, slots)
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        equal(out, want)
        equal(run(), want)
