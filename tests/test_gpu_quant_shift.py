"""Shifted reuse over 8-bit caches, several shifts after each other: the scales
are those of the turned rows, V stays, and K's error grows by the rounding of
each shift and no more."""

import numpy as np
import pytest
import torch

import workloads as W
from oracle import acache_oracle as O
from paper_2608_26140_amd import acache as A
from paper_2608_26140_amd import workload as WL

pytestmark = pytest.mark.gpu


def keys_of(batch, n):
    d = batch.model.dims
    return [t.double().cpu().numpy().reshape(-1, d.n_kv_heads, d.head_dim)
            for t in A.acache_quant_load(d, batch.caches[n], batch.affix_slots)]


@pytest.mark.parametrize("qb,paged", [(64, None), (32, 64), (128, 128)])
def test_scales_follow_the_turned_rows(qb, paged):
    """Every row alike: one pair of K just below a scale's largest value, turned
    by 1 rad (sum of its elements 1.38 times: the scale doubles) and by 10 more
    (11 rad are 3.5 turns of pi: back within it).  All blocks agree, the short
    last one too."""
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=qb, block_size=paged, keep_host=False).batch
    d = batch.model.dims
    assert batch.L % qb
    x = torch.zeros(batch.L, d.n_kv_heads, d.head_dim, device="cuda")
    x[:, :, 0] = x[:, :, d.head_dim // 2] = 0.9 * 448
    rows = x.flatten(1).to(torch.bfloat16)
    for c in batch.caches:
        c.clear()
        A.acache_quant_store(d, c, rows, rows, batch.affix_slots)
    used = -(-batch.L // qb)
    for delta, scale in ((1, 2.0), (10, 1.0), (0, 1.0)):
        batch.shift_affix(delta)
        for c in batch.caches:
            assert (c.k_scales[:used] == scale).all(), delta
            assert (c.v_scales[:used] == 1.0).all()


def test_error_of_several_shifts():
    w = W.get_config("mini-stack")
    batch = WL.build(w, quant_block=64, keep_host=False).batch
    d, N = batch.model.dims, w.dims.n_layers
    before = [keys_of(batch, n) for n in range(N)]
    half = d.head_dim // 2
    # length of a pair's vector: what a turn keeps
    length = [np.hypot(k[..., :half], k[..., half:]) for k, _ in before]
    error = [np.zeros_like(p) for p in length]
    total = 0
    for delta in (37, -37, 111, -50):
        batch.shift_affix(delta)
        total += delta
        for n, (k, v) in enumerate(before):
            k2, v2 = keys_of(batch, n)
            np.testing.assert_array_equal(v, v2)
            want = O.rerotate_keys(k, np.full(len(k), total), d.rope_base)
            sc = batch.caches[n].k_scales[batch.affix_slots.long() // 64].double().cpu().numpy()[..., None]
            # each element is rounded to bf16 and to e4m3 (half a step each; 1e-4: fp32 angles), a pair's two at most
            big = length[n] + error[n]
            error[n] = error[n] + np.sqrt(2) * (np.maximum(2.0 ** -4 * big, 2.0 ** -10 * sc) + 1.1 * 2.0 ** -8 * big + 1e-4)
            got = np.hypot(k2[..., :half] - want[..., :half], k2[..., half:] - want[..., half:])
            print(f"[shift] {total} layer {n}: {float((got / error[n]).max()):.3f} of the bound", flush=True)
            assert (got <= error[n]).all()
