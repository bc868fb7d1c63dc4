"""Every way the attention over an 8-bit cache can take (either kernel, with and
without key splits, both with each limit of what is left), each with ordinary
values, scales at the ends of their range, keys that are all absent, maxima far
apart, and NaN in one key or value.  Bounds as in test_gpu_quant."""

import numpy as np
import pytest
import torch

from paper_2608_26140_amd import acache as A
from tests import quant_reference as Q
from tests.gpu_util import up_i32
from tests.quant_attention_cases import WAYS, cu, way_of
from tests.test_gpu_quant import DEV, Pair, filled, many, sampled

pytestmark = pytest.mark.gpu


def case(way):
    """The batch, a cache for it, its workspace; the library takes this way."""
    _, H, Hkv, rows, keys, ws = WAYS[way]
    p = filled(H, Hkv, 1900, 64, seed=len(way))
    size = A.quant_workspace(p.dims, sum(rows), p.pool).numel() if ws else 0
    assert way_of(p.dims, rows, keys, size) == way
    return p, rows, keys, ws


def queries(p, rows, spread=1.3, seed=1):
    g = torch.Generator(DEV).manual_seed(seed)
    return spread * torch.randn(sum(rows), p.dims.n_heads * 128, device=DEV, generator=g)


@pytest.mark.parametrize("way", WAYS)
def test_ordinary(way):
    p, rows, keys, ws = case(way)
    p.pool.clear(slice(640, 768))  # two empty blocks
    for r in p.ref:
        r.scales[10:12] = 0.0
    slots = p.rng.integers(-40, 1940, sum(keys))
    out, lse = many(p, rows, keys, slots, ws=ws, what=way)
    again = many(p, rows, keys, slots, ws=ws, what=way)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("way", WAYS)
def test_only_absent_keys(way):
    """Every key is zero, and so is every value: zeros, and the logarithm of the number of keys."""
    p, rows, keys, ws = case(way)
    p.pool.clear(slice(64, 128))
    for r in p.ref:
        r.scales[1] = 0.0
    slots = np.resize([-1, 1900, 2 ** 31 - 1, -2 ** 31, 70, 127], sum(keys))
    out, lse = many(p, rows, keys, slots, ws=ws, what=way)
    assert not out.any()


@pytest.mark.parametrize("way", WAYS)
def test_requests_with_and_without_keys_that_are_there(way):
    p, rows, keys, ws = case(way)
    slots = p.rng.integers(0, 1900, sum(keys))
    at = cu(keys)
    for b in range(0, len(keys), 2):  # of every second request one key is there, its last
        slots[at[b]:at[b + 1] - 1] = -1
    many(p, rows, keys, slots, ws=ws, what=way)


@pytest.mark.parametrize("way", WAYS)
def test_extreme_scales(way):
    """Rows and keys as in test_gpu_quant's test of that name."""
    p, rows, keys, ws = case(way)
    n = 1900
    x, v = (p.rng.normal(0, 1, (n, p.Hkv, 128)) for _ in range(2))
    x[:320] *= 1e-36
    x[320:640] *= 1e4
    x[640:960, :, 7] *= 300
    v[320:640] *= 1e-30
    v[960:1280] *= 1e30
    p.store(np.arange(n), x=[x * 1e-4, v], check=False)
    q = queries(p, rows, 1.0)
    q[0::5] *= 1e-3
    q[1::5, ::64] *= 1e4
    q[1::5] *= 1e-4
    q[2::5] = 0.0
    q[3::5] *= 1e-38
    many(p, rows, keys, p.rng.integers(0, n, sum(keys)), q=q.to(torch.bfloat16), ws=ws, what=way)


@pytest.mark.parametrize("way", WAYS)
def test_maxima_far_apart(way):
    """Logits of some hundreds; one key dominates, the first or the last of its
    request: the maximum moves late, or all but one part weigh nothing."""
    p, rows, keys, ws = case(way)
    big = np.full((1, p.Hkv, 128), 40.0)
    p.store([1899], x=[big, big], check=False)
    slots = p.rng.integers(0, 1899, sum(keys))
    at = cu(keys)
    for b in range(len(keys)):
        slots[at[b] if b % 2 else at[b + 1] - 1] = 1899
    many(p, rows, keys, slots, q=queries(p, rows, 20.0).to(torch.bfloat16), ws=ws, what=way)


def run(p, rows, keys, slots, q, ws):
    lse = torch.empty(sum(rows), p.dims.n_heads, device=DEV)
    w = A.quant_workspace(p.dims, sum(rows), p.pool) if ws else None
    out = A.acache_quant_attention(p.dims, cu(rows), cu(keys), q, up_i32(slots), p.pool, lse=lse, ws=w)
    return out.view(sum(rows), p.dims.n_heads, 128), lse


@pytest.mark.parametrize("which", ["K", "V"])
@pytest.mark.parametrize("way", WAYS)
def test_nan_shows_where_it_is_read(way, which):
    """A NaN in one dimension of one head's key makes that head's rows of the
    requests that read it NaN, in a value that dimension of them, and nothing else."""
    p, rows, keys, ws = case(way)
    x = p.rng.normal(0, 1, (1, p.Hkv, 128))
    bad = x.copy()
    bad[0, -1, 3] = np.nan
    p.store([1000], x=[bad, x] if which == "K" else [x, bad], check=False)
    slots = p.rng.integers(0, 1000, sum(keys))
    at, reader = cu(keys), len(keys) // 2
    slots[at[reader] + keys[reader] // 3] = 1000
    out, lse = run(p, rows, keys, slots, queries(p, rows).to(torch.bfloat16), ws)
    want = torch.zeros_like(out, dtype=torch.bool)
    r0, r1, rep = cu(rows)[reader], cu(rows)[reader + 1], p.dims.n_heads // p.Hkv
    if which == "K":
        want[r0:r1, -rep:] = True
    else:
        want[r0:r1, -rep:, 3] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.isfinite(out[~want]).all()
    assert torch.equal(torch.isnan(lse), want.all(-1))


@pytest.mark.parametrize("way", WAYS)
def test_small_values_behind_small_weights(way):
    """Values at the smallest scale, one key of weight 1 and the others of
    about 2^-12 each.  A weight times its scale is a bf16 number (2^-117 is the
    smallest scale): where it is subnormal its rounding, half of 2^-133, adds
    up to 448 times that for each key."""
    p, rows, keys, ws = case(way)
    n = 1900
    k = np.zeros((n, p.Hkv, 128))
    k[n - 1, :, 0] = 1.0
    v = p.rng.uniform(1.0, 2.0, (n, p.Hkv, 128)) * 2.0 ** -110
    p.store(np.arange(n), x=[k, v], check=False)
    assert (p.pool.v_scales == 2.0 ** -117).all()
    q = torch.zeros(sum(rows), p.dims.n_heads * 128, device=DEV)
    q.view(-1, p.dims.n_heads, 128)[:, :, 0] = 94.0  # 94 / sqrt(128) = 12 ln 2
    q = q.to(torch.bfloat16)
    slots = p.rng.integers(0, n - 1, sum(keys))
    for a in cu(keys)[:-1]:
        slots[a] = n - 1
    out, lse = run(p, rows, keys, slots, q, ws)
    worst = 0.0
    for b, pick in enumerate(sampled(cu(rows), 2, p.rng)):
        sl = slots[cu(keys)[b]:cu(keys)[b + 1]]
        q64 = q[torch.from_numpy(pick).to(DEV)].double().cpu().numpy().reshape(len(pick), -1, 128)
        ref, _, weight, big = Q.attention(q64, p.ref[0].values(sl), p.ref[1].values(sl), p.dims.n_heads // p.Hkv)
        got = out[torch.from_numpy(pick).to(DEV)].double().cpu().numpy()
        total = 132 * 2.0 ** -24 * big + (len(sl) + 8) * 2.0 ** -24
        bound = 2.0 ** -8 * (np.abs(ref) + weight) * 1.01 + (2 * total)[..., None] * weight + len(sl) * 448 * 2.0 ** -134
        strict = bound - len(sl) * 448 * 2.0 ** -134
        print(f"[small] {way} request {b}: {(np.abs(got - ref) / bound).max():.3f} of the bound, "
              f"{(np.abs(got - ref) / strict).max():.3f} without the subnormals' part", flush=True)
        worst = max(worst, float((np.abs(got - ref) / bound).max()))
    assert worst <= 1.0
