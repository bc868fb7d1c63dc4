"""The sampled commit against its definition in float64: the same tokens, and their
probabilities."""

import math

import numpy as np
import pytest
import torch

from paper_2608_26140_amd import acache as A
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def check(x, u, t=None, k=None, p=None, m=None, what=""):
    """x [rows, n] on the CPU (any row stride); settings lists or None."""
    rows, n = x.shape
    f = lambda v, dt: None if v is None else torch.tensor(v, dtype=dt)
    t, k, p, m = f(t, F32), f(k, torch.int32), f(p, F32), f(m, F32)
    u = torch.as_tensor(u, dtype=torch.float64)
    base = torch.empty(rows, x.stride(0) if rows > 1 else n, dtype=x.dtype, device="cuda")
    base[:, :n] = x.cuda()
    conf, prob = (torch.full((rows,), math.nan, device="cuda") for _ in range(2))
    ids = torch.full((rows + 3,), -1, dtype=torch.int32, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32) + 2
    pos[0] = rows + 9  # nowhere
    c = lambda v: None if v is None else v.cuda()
    out = A.acache_sample_commit(base[:, :n], u.cuda(), c(t), c(k), c(p), c(m), conf=conf, prob=prob,
                                 commit_pos=pos.cuda(), ids=ids)
    d = lambda v: None if v is None else v.double().numpy()
    got = out.cpu().numpy()
    want, wc, wp = R.sample(x.double().numpy(), u.numpy(), d(t), d(k), d(p), d(m), got)
    bad = np.flatnonzero(got != want)
    assert bad.size == 0, f"{what}: rows {bad[:5]}: {got[bad[:5]]} for {want[bad[:5]]}"
    # conf and prob: quotients of sums in 64 bits (weights to 2^-45, so the kept weight to n 2^-45), rounded to fp32
    assert np.all(np.abs(conf.cpu().numpy() - wc) <= 2.0 ** -23 * wc + 1e-37), what
    assert np.all(np.abs(prob.cpu().numpy() - wp) <= (2.0 ** -23 + n * 2.0 ** -44) * wp + 2.0 ** -44), what
    back = ids.cpu().numpy()
    assert (back[:2] == -1).all() and back[2] == -1 and (back[3:2 + rows] == want[1:]).all() and back[2 + rows] == -1
    # without the optional results, the same tokens; twice, the same bits
    again = A.acache_sample_commit(base[:, :n], u.cuda(), c(t), c(k), c(p), c(m))
    assert torch.equal(again, out)
    return out


def logits(rows, n, dt, seed, spread=2.5, ld=None):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(rows, ld or n, generator=g)
    x[:, torch.randint(n, (min(n, 12),), generator=g)] += 9 * torch.rand(rows, min(n, 12), generator=g)
    return x.to(dt)[:, :n]


def uniform(rows, seed):
    return torch.rand(rows, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("n,ld", [(1, 1), (2, 2), (7, 9), (64, 64), (1000, 1000), (1021, 1021), (1024, 1032), (8192, 8192),
                                  (20011, 20013), (126464, 126464), (131073, 131080), (262144, 262144)])
def test_sizes(dt, n, ld):
    print(f"sample {dt} {n} of {ld}", flush=True)
    rows = 24 if n < 50000 else 6
    x, u = logits(rows, n, dt, n, ld=ld), uniform(rows, n)
    g = np.random.default_rng(n)
    check(x, u, what="no cuts")
    check(x, u, t=g.uniform(0.2, 1.7, rows).tolist(), what="temperature")
    check(x, u, k=g.integers(1, min(n, 300) + 1, rows).tolist(), what="top-k")
    check(x, u, p=g.uniform(0.02, 0.999, rows).tolist(), what="top-p")
    check(x, u, m=g.uniform(0.0005, 0.4, rows).tolist(), what="min-p")
    check(x, u, t=g.uniform(0.4, 1.7, rows).tolist(), k=g.integers(0, min(n, 3000) + 1, rows).tolist(),
          p=g.uniform(0.3, 1.05, rows).tolist(), m=g.uniform(-0.05, 0.05, rows).tolist(), what="all")


@pytest.mark.parametrize("dt", [BF, F32])
def test_ties_are_told_apart_by_index(dt):
    g = torch.Generator().manual_seed(9)
    rows, n = 64, 3001
    x = torch.randint(-2, 3, (rows, n), generator=g).to(dt)
    x[:8] = 0.5  # all alike
    x[8:12] = 0.0
    x[8:12, ::2] = -0.0
    u = uniform(rows, 10)
    check(x, u, what="no cuts")
    check(x, u, k=[1 + 37 * i for i in range(rows)], what="top-k inside ties")
    check(x, u, p=[(i + 0.37) / rows for i in range(rows)], what="top-p inside ties")
    check(x, u, k=[1 + 53 * i for i in range(rows)], p=[(i + 0.37) / rows for i in range(rows)], what="both")
    check(x, u, m=[0.13] * rows, what="min-p")


@pytest.mark.parametrize("dt", [BF, F32])
def test_values_at_the_ends(dt):
    """NaN, infinities, the type's lowest value in masked places, tiny and huge logits, rows with nothing to draw."""
    n, inf, nan = 517, math.inf, math.nan
    lowest, tiny = torch.finfo(dt).min, 1e-38
    x = logits(16, n, dt, 3).clone()
    x[0, ::2] = nan
    x[1, 1:] = -inf
    x[2] = -inf
    x[3] = nan
    x[4] = nan
    x[4, 100:] = -inf
    x[5, [7, 300]] = inf
    x[6, 5:] = lowest
    x[7] = lowest
    x[8] = torch.linspace(-1, 1, n).to(dt) * tiny
    x[9] = torch.linspace(-1, 1, n).to(dt) * 1e38
    x[10, ::3] = torch.tensor(1e-30).to(dt)
    x[11] = torch.linspace(900, 1100, n).to(dt)
    x[12, 3] = 5000.0
    x[13] = torch.linspace(-1100, -1000, n).to(dt)
    x[14, 2:] = -1e30
    x[15, 1:] = nan
    for u in (0.0, 0.3, 0.77, 1.0 - 2.0 ** -53):
        us = [u] * 16
        check(x, us, what=f"u {u}")
        check(x, us, t=[0.7] * 16, k=[40] * 16, p=[0.9] * 16, what=f"u {u}, top-k and top-p")
        check(x, us, t=[1e30] * 16, p=[0.6] * 16, what=f"u {u}, all but equal weights")
        check(x, us, m=[0.05] * 16, k=[500] * 16, what=f"u {u}, min-p")


@pytest.mark.parametrize("dt", [BF, F32])
def test_logits_next_to_zero(dt):
    """A few of them beside ordinary ones, many, the largest among them, and a border between them."""
    n = 3001
    g = torch.Generator().manual_seed(8)
    tiny = torch.tensor([1e-10, -1e-12, 3e-9, -2e-38, 1e-30, 7e-9, -6e-9, 1e-20, -1e-20, 2e-39])
    at = lambda count: torch.randperm(n, generator=g)[:count]
    x = logits(8, n, F32, 9).clone()
    x[0, at(10)] = tiny
    x[1, at(20)] = tiny.repeat(2)
    x[2] = -x[2].abs()
    x[2, at(10)] = -tiny.abs()
    x[2, at(5)] = 0.0
    x[3] = -x[3].abs()
    x[3, at(10)] = tiny
    x[4] = -x[4].abs() - 1
    x[4, at(2000)] = 0.0
    x[4, at(10)] = tiny
    x[5] = tiny[torch.randint(10, (n,), generator=g)]
    x[5, at(1000)] = 0.0
    x[6, at(1)] = 1e-10
    x[6, at(800)] = -0.0
    x[7, at(16)] = tiny[torch.randint(10, (16,), generator=g)]
    x = x.to(dt)
    rows = x.repeat(5, 1)
    us = [u for u in (0.0, 0.2, 0.5, 0.9, 1.0 - 2.0 ** -53) for _ in range(8)]
    check(rows, us, what="as they are")
    check(rows, us, t=[0.8] * 40, k=[1500] * 40, p=[0.9] * 40, what="top-k and top-p")
    check(rows, us, t=[3.0] * 40, m=[0.3] * 40, what="min-p")
    check(rows, us, t=[50.0] * 40, k=[2010] * 40, what="all but equal weights, top-k")


@pytest.mark.parametrize("dt", [BF, F32])
def test_settings_at_their_ends(dt):
    inf, nan = math.inf, math.nan
    x = logits(9, 1500, dt, 4)
    u = uniform(9, 5)
    greedy = x.double().argmax(1)
    for t in ([0.0] * 9, [-1.0] * 9, [nan] * 9):
        out = check(x, u, t=t, what=f"temperature {t[0]}")
        assert torch.equal(out.cpu().long(), greedy)
    check(x, u, t=[inf, 1e-30, 1e-45, 3e38, 1e-3, 0.01, 50.0, 1e6, 1.0], what="temperatures")
    check(x, u, k=[0, -1, 1, 2, 1499, 1500, 1501, 2 ** 31 - 1, -2 ** 31], what="top-k")
    check(x, u, p=[0.0, -1.0, nan, 1.0, 1.5, 1e-30, 1 - 2.0 ** -24, inf, -inf], what="top-p")
    check(x, u, m=[0.0, -1.0, nan, 1.0, 1.5, 1e-30, 1 - 2.0 ** -24, inf, 1e-45], what="min-p")
    check(x, [0.0, -1.0, nan, 1.0, 1.5, inf, -inf, 2.0 ** -1074, 1 - 2.0 ** -53], what="u")


def test_greedy_rows_agree_with_the_argmax():
    x = logits(40, 5003, BF, 6).cuda()
    conf, conf2, prob = (torch.empty(40, device="cuda") for _ in range(3))
    a = A.acache_argmax_commit(x, conf=conf)
    b = A.acache_sample_commit(x, torch.rand(40, dtype=torch.float64, device="cuda"), torch.zeros(40, device="cuda"),
                               conf=conf2, prob=prob)
    assert torch.equal(a, b) and (prob == 1).all()
    assert torch.allclose(conf, conf2, rtol=1e-5)


def test_frequencies_follow_the_probabilities():
    """Evenly spaced u over many rows of one distribution: each token as often as its probability says."""
    rows, n = 4096, 50
    row = logits(1, n, F32, 7)
    x = row.expand(rows, n).contiguous().cuda()
    u = ((torch.arange(rows, dtype=torch.float64) + 0.5) / rows).cuda()
    out = A.acache_sample_commit(x, u, torch.full((rows,), 1.3, device="cuda"))
    p = torch.softmax(row.double()[0] / 1.3, 0)
    count = torch.bincount(out.cpu().long(), minlength=n).double()
    assert (count - rows * p).abs().max() <= 1.0 + 1e-6
