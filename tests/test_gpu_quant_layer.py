"""Layers, probe, refresh and decode steps over 8-bit caches.

Teacher-forced layer by layer: the reference takes a layer's bf16 input rows
and the view of the layer's own cache as it stands after the layer (which is
what its attention read: rows are stored first), computes the layer in float64
and is compared with the layer's output under the gate of the bf16 layers.
The stored entries are compared with the reference's K and V: half a step of
e4m3 (2^-4 of the entry, or 2^-10 of the scale where it is subnormal) beside
the error of the bf16 projections."""

import numpy as np
import pytest
import torch

import workloads as W
from oracle import acache_oracle as O
from paper_2608_26140_amd import acache as A
from paper_2608_26140_amd import driver as D
from paper_2608_26140_amd import workload as WL
from tests.gpu_util import TOL, assert_close, up_i32
from tests.oracle_side import anchor_count, oracle_dims

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def view_of(batch, n, slots):
    """float64 K and V [len(slots), H_kv, d_h] of layer n's cache."""
    d = batch.model.dims
    k, v = A.acache_quant_load(d, batch.caches[n], slots)
    return tuple(f64(t).reshape(-1, d.n_kv_heads, d.head_dim) for t in (k, v))


def layers_of(w, s):
    dims = oracle_dims(w)
    return dims, [O.layer_from_bits(b, dims, w.dims.dtype) for b in s.host["layers"]]


def check_layer(w, dims, layer, x, pos, view, out, what):
    """One request's rows through one layer over a given view."""
    q = O.layer_queries(layer, dims, x, pos)
    o, _ = O.attention(q, *view)
    y = x + o.reshape(len(x), -1) @ layer.wo.T
    h = O.rms_norm(y, layer.g2, dims.rms_eps)
    y = y + (O.silu(h @ layer.wg.T) * (h @ layer.wu.T)) @ layer.wd.T
    assert_close(out, y, w.dims.dtype, what)
    return q


def check_stored(dims, layer, x, pos, got, scale_of_row, what):
    for g, ref, name in zip(got, O.layer_kv(layer, dims, x, pos), "KV"):
        near = TOL["bf16"] * np.maximum(np.abs(ref), np.sqrt(np.mean(ref * ref)))  # the projection's error
        step = np.maximum(2.0 ** -4 * (np.abs(ref) + near), 2.0 ** -10 * scale_of_row)
        worst = float((np.abs(g - ref) / (step + near)).max())
        print(f"[stored] {what} {name}: {worst:.3f} of the bound", flush=True)
        assert worst <= 1.0


@pytest.mark.parametrize("name,qb,paged", [("mini-stack", 16, None), ("mini-gqa-infix", 64, None),
                                           ("mini-affix64", 32, 64), ("mini-infix64", 64, 128)])
@pytest.mark.parametrize("norm", [A.ACACHE_NORM_AFFIX, A.ACACHE_NORM_FULL])
def test_probe_and_refresh_layer_by_layer(name, qb, paged, norm):
    w = W.get_config(name)
    s = WL.build(w, quant_block=qb, block_size=paged)
    batch, (dims, layers), N = s.batch, layers_of(w, s), w.dims.n_layers
    S, L, lay = w.layout.seq_len, w.layout.affix_len, w.layout
    ins, scores_at = [], []

    def hook(n, x, scores):
        ins.append(f64(x))
        scores_at.append(f64(scores))
    scores, x, m = batch.probe(norm, layer_hook=hook)
    torch.cuda.synchronize()
    P = S - L
    rows = np.array(lay.nonaffix_positions())
    read = m["read_slots"].view(batch.B, S)
    masked = np.searchsorted(rows, np.array(lay.masked_positions()))
    total = np.zeros((batch.B, L))
    for n in range(N):
        ref = np.zeros((batch.B, L))
        for b in range(batch.B):
            view = view_of(batch, n, read[b].contiguous())
            xi = ins[n][b * P:(b + 1) * P]
            q = check_layer(w, dims, layers[n], xi, rows, view, ins[n + 1][b * P:(b + 1) * P], f"probe {n} request {b}")
            ka = view[0][:L]  # the probe reads the affix first
            lse = O.attention(q, *view)[1] if norm == A.ACACHE_NORM_FULL else None
            for h in range(dims.n_heads):
                logit = q[masked, h] @ ka[:, h // (dims.n_heads // dims.n_kv_heads)].T / np.sqrt(dims.head_dim)
                z = lse[masked, h][:, None] if lse is not None else np.log(np.exp(logit).sum(1, keepdims=True))
                ref[b] += np.exp(logit - z).sum(0)
        got = scores_at[n + 1] - scores_at[n] if n else scores_at[1]
        assert_close(got, ref, "bf16", f"scores of layer {n}")
        total += ref
    assert_close(f64(scores), total, "bf16", "scores")

    k = anchor_count(w)
    anchors = A.acache_topk(scores, k)
    ins.clear()
    y, m = batch.refresh(anchors, k, layer_hook=lambda n, xx: ins.append(f64(xx)))
    torch.cuda.synchronize()
    R = k + S - L
    pos = f64(m["row_pos"]).astype(int).reshape(batch.B, R)
    for n in range(N):
        for b in range(batch.B):
            view = view_of(batch, n, m["read_slots"].view(batch.B, S)[b].contiguous())
            xi, at = ins[n][b * R:(b + 1) * R], slice(b * R, (b + 1) * R)
            check_layer(w, dims, layers[n], xi, pos[b], view, ins[n + 1][at], f"refresh {n} request {b}")
            slots = m["write_slots"][at].contiguous()
            sc = torch.maximum(batch.caches[n].k_scales, batch.caches[n].v_scales)[slots.long() // qb]
            check_stored(dims, layers[n], xi, pos[b], view_of(batch, n, slots), f64(sc)[..., None],
                         f"refresh {n} request {b}")


def test_layer_stores_what_a_store_of_its_rows_does():
    """The cache after a layer, bit for bit, is the cache after storing the K
    and V that the bf16 layer leaves in its pools."""
    w = W.get_config("mini-stack")
    s8, s16 = WL.build(w, quant_block=32), WL.build(w)
    for b in (s8.batch, s16.batch):
        b.maps_ = b.maps(None, 0)
    b8, b16 = s8.batch, s16.batch
    m8, m16 = b8.maps_, b16.maps_
    before = A.QuantPool(*(t.clone() for t in (b8.caches[0].k_codes, b8.caches[0].v_codes, b8.caches[0].k_scales,
                                               b8.caches[0].v_scales)), 32)
    x8, x16 = b8.gather_inputs(m8), b16.gather_inputs(m16)
    P, S, B = b8.S - b8.L, b8.S, b8.B
    cu_rows, cu_keys = [b * P for b in range(B + 1)], [b * S for b in range(B + 1)]
    b8.recompute_layer(0, cu_rows, cu_keys, x8, m8["row_pos"], m8["write_slots"], m8["read_slots"])
    b16.recompute_layer(0, cu_rows, cu_keys, x16, m16["row_pos"], m16["write_slots"], m16["read_slots"])
    at = m16["write_slots"].long()
    A.acache_quant_store(b8.model.dims, before, b16.k_pools[0][at], b16.v_pools[0][at], m8["write_slots"])
    for a, b in zip((before.k_scales, before.v_scales), (b8.caches[0].k_scales, b8.caches[0].v_scales)):
        assert torch.equal(a, b)
    everything = torch.arange(b8.n_slots, dtype=torch.int32, device="cuda")
    for a, b in zip(A.acache_quant_load(b8.model.dims, before, everything),
                    A.acache_quant_load(b8.model.dims, b8.caches[0], everything)):
        assert torch.equal(a, b)


def test_decode_steps_layer_by_layer():
    """Two decode steps of a block: its rows overwrite their slots, and every
    other entry keeps its value up to the rounding to a raised scale."""
    w = W.get_config("mini-serve")
    s = WL.build(w, quant_block=16)
    batch, (dims, layers), N, B = s.batch, layers_of(w, s), w.dims.n_layers, w.batch
    k, blen = anchor_count(w), w.decode_block
    anchors, _ = batch.select_anchors(k)
    _, m = batch.refresh(anchors, k)
    plan = D.DecodePlan(batch, k, blen, w.layout.mask_len // blen, full=False)
    S, d = w.layout.seq_len, batch.model.dims
    for blk in (0, 2):
        wslots = plan.write_slots(batch, blk)
        before = [view_of(batch, n, m["read_slots"]) for n in range(N)]
        h = A.acache_gather_rows(batch.x_src, plan.pos[blk], batch.remap)
        cu_rows, cu_keys = [b * blen for b in range(B + 1)], [b * S for b in range(B + 1)]
        pos = f64(plan.row_pos[blk]).astype(int).reshape(B, blen)
        for n in range(N):
            x = f64(h)
            batch.recompute_layer(n, cu_rows, cu_keys, h, plan.row_pos[blk], wslots, m["read_slots"])
            torch.cuda.synchronize()
            view = view_of(batch, n, m["read_slots"])
            written = np.isin(m["read_slots"].cpu().numpy(), wslots.cpu().numpy())
            sc = torch.maximum(batch.caches[n].k_scales, batch.caches[n].v_scales)[m["read_slots"].long() // 16]
            step = f64(sc)[..., None] * 2.0 ** -10
            for a, b in zip(before[n], view):
                assert np.all(np.abs(a - b)[~written] <= step[~written])
            for b in range(B):
                at, keys = slice(b * blen, (b + 1) * blen), slice(b * S, (b + 1) * S)
                check_layer(w, dims, layers[n], x[at], pos[b], tuple(t[keys] for t in view), f64(h)[at],
                            f"block {blk} layer {n} request {b}")
        again = D.decode_step(batch, plan, blk, m, anchors)  # the same ids: the same rows
        assert torch.equal(again, h)


def run_chain(batch, w):
    k = anchor_count(w)
    anchors, scores = batch.select_anchors(k)
    x, _ = batch.refresh(anchors, k)
    return anchors, scores, x


def test_paged_plan_is_the_flat_plan():
    """Blocks of slots are whole blocks of scales: the same bits either way."""
    w = W.get_config("mini-affix64")
    flat, paged = (WL.build(w, quant_block=32, block_size=bs).batch for bs in (None, 64))
    for a, b in zip(run_chain(flat, w), run_chain(paged, w)):
        assert torch.equal(a, b)
    assert paged.kv_bytes(3) == 3 * (64 * paged.model.kv_width + 2 * paged.model.dims.n_kv_heads * 4) * 2 * w.dims.n_layers


def test_captured_chain():
    """Probe, selection and refresh replayed from a graph, eager runs between."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64, keep_host=False).batch
    run_chain(batch, w)
    ref = [t.clone() for t in run_chain(batch, w)]  # scales have seen all rows
    graph, out = D.capture(lambda: run_chain(batch, w))
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, out))
        assert all(torch.equal(a, b) for a, b in zip(ref, run_chain(batch, w)))


def test_shifted_affix():
    """The affix's K turned by a position delta: the turned values, rounded
    again; V keeps its values."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64, keep_host=False).batch
    d = batch.model.dims
    before = [view_of(batch, n, batch.affix_slots) for n in range(w.dims.n_layers)]
    batch.shift_affix(37)
    for n, (k, v) in enumerate(before):
        k2, v2 = view_of(batch, n, batch.affix_slots)
        np.testing.assert_array_equal(v, v2)
        want = O.rerotate_keys(k, np.full(len(k), 37), d.rope_base)
        sc = f64(batch.caches[n].k_scales[batch.affix_slots.long() // 64])[..., None]
        # the turned value is rounded to bf16, then to e4m3
        bound = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * sc) + 1.1 * 2.0 ** -8 * np.abs(want) + 1e-4
        assert np.all(np.abs(k2 - want) <= bound)


def test_schedules_run_and_agree():
    """tau = 0 commits a block at once: the one-step schedule's ids."""
    w = W.get_config("mini-serve")
    k, blen, n_blocks = anchor_count(w), w.decode_block, w.layout.mask_len // w.decode_block
    got = []
    for threshold in (False, True):
        s = WL.build(w, quant_block=64, keep_host=False)
        batch = s.batch
        g = torch.Generator(device="cuda").manual_seed(3)
        head = D.Head(torch.ones(w.dims.d_model, dtype=torch.bfloat16, device="cuda"),
                      torch.randn(w.dims.vocab, w.dims.d_model, generator=g, device="cuda").to(torch.bfloat16))
        plan = D.DecodePlan(batch, k, blen, n_blocks, full=False)
        if threshold:
            assert D.decode_threshold_schedule(batch, head, plan, k, 0.0) == [1] * n_blocks
        else:
            logits = torch.empty((batch.B * blen, w.dims.vocab), dtype=torch.bfloat16, device="cuda")
            committed = torch.empty((n_blocks, batch.B * blen), dtype=torch.int32, device="cuda")
            D.decode_schedule(batch, head, plan, k, logits, committed)
        torch.cuda.synchronize()
        got.append(batch.remap.clone())
    assert torch.equal(*got)


def test_refusals():
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64, keep_host=False).batch
    with pytest.raises(ValueError):
        batch.select_anchors_hkvd(4)
    with pytest.raises(ValueError):
        WL.build(w, quant_block=64, block_size=96, keep_host=False)
    with pytest.raises(ValueError):
        WL.build(W.get_config("tiny-f32"), quant_block=64, keep_host=False)
    d, m = batch.model.dims, batch.maps(None, 0)
    x = batch.gather_inputs(m)
    P, S = batch.S - batch.L, batch.S
    with pytest.raises(A.AcacheError) as e:  # a workspace without the 8-bit regions
        A.acache_quant_layer_recompute(d, batch.model.lw[0], [0, P], [0, S], x, m["row_pos"], m["write_slots"],
                                       m["read_slots"], batch.caches[0], A.workspace(d, P, 1, 0))
    assert e.value.status == 5
