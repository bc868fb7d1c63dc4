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


@pytest.mark.parametrize("name,qb,paged", PLANS)
def test_affix_materialised_anew(name, qb, paged):
    """A second affix in the slots of a first, larger one; the donor's other
    rows in slots of large rows."""
    w = W.get_config(name)
    fresh, used = (WL.build(w, quant_block=qb, block_size=paged).batch for _ in range(2))
    occupy(used, np.arange(used.n_slots))
    S, L, ab = fresh.S, fresh.L, fresh.ab
    got = []
    for b in (fresh, used):
        slots = np.empty(S, dtype=np.int64)
        inside = (np.arange(S) >= ab) & (np.arange(S) < ab + L)
        slots[inside] = b.affix_slots.cpu().numpy()
        slots[~inside] = b.private_slots(S - L)[-1]
        slots = up_i32(slots)
        g = torch.Generator(device="cuda").manual_seed(4)
        x = torch.randn(S, w.dims.d_model, generator=g, device="cuda").to(torch.bfloat16)
        b.materialize_affix(x, up_i32(np.arange(S)), slots, slots)
        got.append([x, *(t for c in b.caches for t in A.acache_quant_load(b.model.dims, c, b.affix_slots))])
    equal(got[1], got[0])
    equal(chain(used, w), chain(fresh, w))


def test_affix_materialised_in_parts():
    """A call that writes some of the affix's rows keeps the others."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64).batch
    dims, c = batch.model.dims, batch.caches[0]
    kept = batch.affix_slots[:-10].contiguous()
    before = A.acache_quant_load(dims, c, kept)
    x = torch.randn(10, w.dims.d_model, device="cuda").to(torch.bfloat16)
    # write slots outside the cache are skipped, here as in every call
    slots = torch.cat([batch.affix_slots[-8:], up_i32([-1, batch.n_slots])])
    batch.materialize_affix(x, up_i32(np.arange(batch.L - 10, batch.L)), slots, batch.affix_slots)
    after = A.acache_quant_load(dims, c, kept)
    for a, b, s in zip(before, after, (c.k_scales, c.v_scales)):
        step = s[kept.long() // 64].repeat_interleave(dims.head_dim, 1)
        # at most rounded to the scale that the new rows need: half a step of e4m3 each
        assert ((a.float() - b.float()).abs() <= torch.maximum(2.0 ** -4 * a.float().abs(), 2.0 ** -10 * step)).all()
        assert b[-2:].any()


def test_parts_keep_the_other_rows_of_their_blocks():
    """Rows written part by part, some outside the affix: a part leaves what the
    parts before it stored in the same private block."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64).batch
    dims, c = batch.model.dims, batch.caches[0]
    own = up_i32(batch.private_slots(60)[1])
    first, second = own[:25].contiguous(), torch.cat([own[25:], batch.affix_slots[:20]])
    for slots in (first, second):
        x = torch.randn(len(slots), w.dims.d_model, device="cuda").to(torch.bfloat16)
        batch.materialize_affix(x, up_i32(np.arange(len(slots))), slots, batch.affix_slots)
    k, v = A.acache_quant_load(dims, c, own)
    assert k.any(1).all() and v.any(1).all()


def test_affix_materialised_in_a_graph():
    """Captured and replayed over large earlier rows: the eager call's bits."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64).batch
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = torch.randn(batch.L, w.dims.d_model, generator=g, device="cuda").to(torch.bfloat16)
    x, pos = torch.empty_like(rows), up_i32(np.arange(batch.L))

    def run():
        x.copy_(rows)
        batch.materialize_affix(x, pos, batch.affix_slots, batch.affix_slots)
        return [x, *(t for c in batch.caches for t in A.acache_quant_load(batch.model.dims, c, batch.affix_slots))]
    want = [t.clone() for t in run()]
    graph, out = D.capture(run)
    for _ in range(3):
        occupy(batch, np.arange(batch.n_slots))
        graph.replay()
        torch.cuda.synchronize()
        equal(out, want)
        occupy(batch, np.arange(batch.n_slots))
        equal(run(), want)
