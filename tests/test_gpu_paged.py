"""The cache in blocks: append and attention against plain float64, element by element
within the bounds of their roundings (tests/paged_reference.py)."""

import math

import pytest
import torch

from paper_2608_26140_amd import acache as A
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAME = {BF: "bf16", F32: "f32"}


def dims_of(H, G, d, dt, base=10000.0):
    return A.make_dims(H * d, H, G, d, 256, NAME[dt], rope_base=base)


def pools(n_slots, width, dt, ld=None, seed=0):
    """K and V of n_slots rows, `width` wide, in a wider allocation if ld is given (CPU)."""
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n_slots, ld or width, generator=g).to(dt)[:, :width] for _ in range(2)]


def some_tables(batch, max_blocks, n_blocks, seed=1):
    g = torch.Generator().manual_seed(seed)
    assert batch * max_blocks <= n_blocks
    return torch.randperm(n_blocks, generator=g)[:batch * max_blocks].view(batch, max_blocks).to(torch.int32)


def up(t):
    """To the device, keeping the strides of a view."""
    if t.dim() == 2 and not t.is_contiguous():
        base = torch.empty(t.shape[0], t.stride(0), dtype=t.dtype, device="cuda")
        base[:, :t.shape[1]] = t.cuda()
        return base[:, :t.shape[1]]
    return t.cuda()


def check(got, ref, bound, what):
    got = got.double().cpu()
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    off = torch.where(same, 0.0, (got - ref).abs())
    bad = ~(same | (off <= bound))
    print(f"{what}: largest error {float(off[~bad].max()) if (~bad).any() else 0:.3e}, "
          f"at most {float(torch.where(bound > 0, off / bound, 0.0)[~bad].max()) if (~bad).any() else 0:.2f} of its bound", flush=True)
    assert not bad.any(), f"{what}: {int(bad.sum())} elements off, first {got[bad][0]} for {ref[bad][0]} ({bound[bad][0]})"


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("dt,H,G,d,batch,per,block,max_blocks,first,base", [
    (BF, 4, 4, 128, 1, 1, 64, 3, 5, 10000.0),
    (BF, 28, 4, 128, 3, 7, 16, 4, 0, 10000.0),
    (BF, 8, 1, 128, 2, 5, 1, 30, 3, 500000.0),
    (BF, 32, 32, 128, 1, 33, 24, 5, 61, 10000.0),
    (BF, 2, 2, 128, 1, 2100, 256, 9, 100, 10000.0),  # the many-row launch
    (F32, 4, 2, 32, 2, 9, 16, 3, 11, 10000.0),
    (F32, 3, 1, 6, 2, 5, 7, 4, 2, 10000.0),          # rows of no whole 16 bytes
    (F32, 2, 2, 128, 1, 2050, 128, 17, 3, 10000.0),
])
def test_append(dt, H, G, d, batch, per, block, max_blocks, first, base):
    print(f"append {dt} {H}/{G} x {d}, {batch} x {per}, block {block}", flush=True)
    g = torch.Generator().manual_seed(3)
    n = batch * per
    n_blocks = batch * max_blocks + 2
    kp, vp = pools(n_blocks * block + 1, G * d, dt, seed=5)
    tables = some_tables(batch, max_blocks, n_blocks)
    tables[0, max_blocks - 1] = -1  # nobody's
    if batch > 1:
        tables[1, max_blocks - 1] = n_blocks
    qkv = torch.randn(n, (H + 2 * G) * d, generator=g).to(dt)
    at = (first + torch.arange(per)).repeat(batch)
    pos = (at + 1000 * torch.arange(batch).repeat_interleave(per)).to(torch.int32)
    at = at.to(torch.int32)
    if per > 3:
        pos[1] = -1                        # padding
        at[2], at[3] = -5, max_blocks * block  # no slot
    dims = dims_of(H, G, d, dt, base)
    kd, vd, x, td = up(kp), up(vp), up(qkv), tables.cuda()
    cache = A.PagedCache(kd, vd, block, td)
    q, k, v = x.split([H * d, G * d, G * d], 1)
    q_out = A.acache_paged_append(dims, cache, k, v, pos.cuda(), per, at=at.cuda(), q=q)
    half = R.HALF[dt]
    kref, kb, vref = kp.double().clone(), torch.zeros(kp.shape, dtype=torch.float64), vp.clone()
    qref, qb = torch.zeros(n, H * d, dtype=torch.float64), torch.zeros(n, H * d, dtype=torch.float64)
    for m in range(n):
        if pos[m] < 0:
            continue
        xq, xk = qkv[m, :H * d].double().view(H, d), qkv[m, H * d:(H + G) * d].double().view(G, d)
        turned = R.rotate(xq, int(pos[m]), base)
        qref[m], qb[m] = turned.flatten(), R.rotate_bound(xq, turned, half).flatten()
        s = R.slot(tables, n_blocks, block, m // per, int(at[m]))
        if s is not None:
            turned = R.rotate(xk, int(pos[m]), base)
            kref[s], kb[s] = turned.flatten(), R.rotate_bound(xk, turned, half).flatten()
            vref[s] = qkv[m, (H + G) * d:]
    check(q_out, qref, qb, "q")
    check(kd, kref, kb, "k pool")
    assert torch.equal(vd.cpu(), vref)
    # in place, and without queries: the same
    k2, v2 = up(kp), up(vp)
    cache2 = A.PagedCache(k2, v2, block, td)
    assert A.acache_paged_append(dims, cache2, k, v, pos.cuda(), per, at=at.cuda()) is None
    assert torch.equal(k2, kd) and torch.equal(v2, vd)
    A.acache_paged_append(dims, cache2, k, v, pos.cuda(), per, at=at.cuda(), q=q, q_out=q)
    assert torch.equal(q, q_out) and torch.equal(k2, kd)


def test_append_far_positions_and_strided_pools():
    dt, H, G, d, block = BF, 2, 2, 128, 16
    kp, vp = pools(64, G * d, dt, ld=G * d + 64, seed=8)
    kd, vd = up(kp), up(vp)
    assert kd.stride(0) == G * d + 64
    tables = torch.full((1, 140000), -1, dtype=torch.int32)
    pos = torch.tensor([2_000_003, 2_000_004, 77], dtype=torch.int32)
    for i, p in enumerate(pos.tolist()):
        tables[0, p // block] = i
    tables[0, 2_000_004 // block] = tables[0, 2_000_003 // block]
    x = torch.randn(3, 2 * G * d, generator=torch.Generator().manual_seed(2)).to(dt)
    dims = dims_of(H, G, d, dt)
    xd = x.cuda()
    A.acache_paged_append(dims, A.PagedCache(kd, vd, block, tables.cuda()), xd[:, :G * d], xd[:, G * d:], pos.cuda(), 3)
    kref, kb, vref = kp.double().clone(), torch.zeros(kp.shape, dtype=torch.float64), vp.clone()
    for m, p in enumerate(pos.tolist()):
        s = R.slot(tables, 4, block, 0, p)
        xk = x[m, :G * d].double().view(G, d)
        t = R.rotate(xk, p, 10000.0)
        kref[s], kb[s], vref[s] = t.flatten(), R.rotate_bound(xk, t, 2.0 ** -8).flatten(), x[m, G * d:]
    check(kd, kref, kb, "k pool")
    assert torch.equal(vd.cpu(), vref)


# ---------------------------------------------------------------- attention
def run_attention(dt, H, G, d, batch, per, block, key_len, ld=None, poison=True, ws="all", tables=None, kv=None, q=None,
                  strided=False, max_len=0):
    key_len = torch.tensor(key_len, dtype=torch.int32)
    longest = max(1, int(key_len.max()))
    max_blocks = -(-longest // block) + 1
    n_blocks = batch * max_blocks + 2
    if tables is None:
        tables = some_tables(batch, max_blocks, n_blocks)
    kp, vp = kv if kv is not None else pools(n_blocks * block, G * d, dt, ld=ld, seed=11)
    if poison:  # nothing but the attended positions holds numbers
        used = torch.zeros(kp.shape[0], dtype=torch.bool)
        for b in range(batch):
            for p in range(max(0, int(key_len[b * per:(b + 1) * per].max())) if per else 0):
                s = R.slot(tables, n_blocks, block, b, p)
                if s is not None:
                    used[s] = True
        kp[~used], vp[~used] = math.nan, math.inf
    if q is None:
        q = torch.randn(batch * per, H * d + (8 if strided else 0), generator=torch.Generator().manual_seed(4)).to(dt)[:, :H * d]
    dims = dims_of(H, G, d, dt)
    cache = A.PagedCache(up(kp), up(vp), block, tables.cuda())
    lse = torch.empty(batch * per, H, device="cuda")
    out = None
    if strided:
        wide = torch.full((batch * per, H * d + 16), 7.0, dtype=dt, device="cuda")
        out = wide[:, :H * d]
    w = None
    if ws != "none":
        size = A.acache_paged_workspace_size(dims, cache, per, max_len)
        w = torch.full((size if ws == "all" else size // ws // 16 * 16,), 255, dtype=torch.uint8, device="cuda")
    got = A.acache_paged_attention(dims, cache, up(q), key_len.cuda(), per, max_len=max_len, out=out, lse=lse, ws=w)
    if strided:
        assert (wide[:, H * d:] == 7.0).all()
    ref = R.attention(q, key_len, kp, vp, block, tables, H, G, d, per)
    check(got, ref[0], ref[2], "out")
    check(lse, ref[1], ref[3], "lse")
    return got, lse


SHAPES = [(BF, 4, 4, 128), (BF, 28, 4, 128), (BF, 8, 1, 128), (F32, 4, 2, 32), (F32, 3, 3, 6), (F32, 5, 1, 128)]


@pytest.mark.parametrize("dt,H,G,d", SHAPES)
@pytest.mark.parametrize("block", [1, 16, 24, 64])
def test_one_token(dt, H, G, d, block):
    print(f"one token {dt} {H}/{G} x {d}, block {block}", flush=True)
    run_attention(dt, H, G, d, 10, 1, block, [0, 1, 2, 31, 32, 33, 128, 129, 257, 500])


@pytest.mark.parametrize("dt,H,G,d", SHAPES)
@pytest.mark.parametrize("per,causal", [(2, True), (5, True), (9, False), (33, True), (40, False)])
def test_rows(dt, H, G, d, per, causal):
    print(f"rows {dt} {H}/{G} x {d}, {per} rows, causal {causal}", flush=True)
    lens = [n - (per - 1 - i) if causal else n for n in (per, 95, 300) for i in range(per)]
    run_attention(dt, H, G, d, 3, per, 16, lens, strided=True)


@pytest.mark.parametrize("H,G,per", [(28, 4, 10), (28, 4, 32), (8, 1, 17), (4, 4, 130), (28, 4, 19)])
@pytest.mark.parametrize("block,causal", [(16, True), (64, False), (48, True)])
def test_many_rows(H, G, per, block, causal):
    """Tiles of 32 and of 128 queries: whole ones and parts of one, waves without any."""
    print(f"many rows {H}/{G}, {per} rows, block {block}, causal {causal}", flush=True)
    lens = [n - (per - 1 - i) if causal else n for n in (max(per, 200), max(per, 333)) for i in range(per)]
    run_attention(BF, H, G, 128, 2, per, block, lens, strided=True)


@pytest.mark.parametrize("per", [25, 40])
def test_many_rows_of_any_lengths(per):
    g = torch.Generator().manual_seed(16)
    lens = torch.randint(0, 300, (3 * per,), generator=g)
    lens[::7] = 0
    lens[per:2 * per] = 0
    run_attention(BF, 28, 4, 128, 3, per, 32, lens.tolist())


@pytest.mark.parametrize("per", [20, 32])
@pytest.mark.parametrize("ws", ["none", 3, "all"])
def test_many_rows_split(ws, per):
    run_attention(BF, 28, 4, 128, 1, per, 16, [1500 + i for i in range(per)], ws=ws)


@pytest.mark.parametrize("per", [20, 30])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_odd_numbers_beside_many_rows(bad, per):
    """As below, with tiles of 32 and of 128 queries, entries without a block among them."""
    H, G, d = 28, 4, 128
    tables = torch.tensor([[6, 2, -1, 0, 3, 7, 1, 99]], dtype=torch.int32)
    lens = [100 + i % 20 for i in range(per)]
    lens[4], lens[9] = 3, 0
    kp, vp = pools(8 * 16, G * d, BF, seed=21)
    vp[R.slot(tables, 8, 16, 0, 110), 1] = bad
    vp[R.slot(tables, 8, 16, 0, 105), G * d - 1] = bad
    vp[R.slot(tables, 8, 16, 0, 50), 7] = bad
    kp[R.slot(tables, 8, 16, 0, 109), :d] = bad
    run_attention(BF, H, G, d, 1, per, 16, lens, tables=tables, kv=(kp, vp), poison=False)


@pytest.mark.parametrize("dt,H,G,d", [SHAPES[1], SHAPES[3]])
def test_rows_of_any_lengths(dt, H, G, d):
    """Every row a length of its own, empty ones and negative ones among them."""
    g = torch.Generator().manual_seed(6)
    lens = torch.randint(0, 400, (4 * 13,), generator=g)
    lens[::5] = 0
    lens[3], lens[17], lens[30] = -7, 1, 2
    lens[13:26] = 0  # a request without any
    run_attention(dt, H, G, d, 4, 13, 32, lens.tolist())


@pytest.mark.parametrize("dt,H,G,d", [SHAPES[0], SHAPES[2], SHAPES[4]])
@pytest.mark.parametrize("ws", ["none", 2, 3, "all"])
def test_splits(dt, H, G, d, ws):
    """The same call with any workspace; a given max_len only moves the splits."""
    print(f"splits {dt} {H}/{G} x {d}, workspace {ws}", flush=True)
    run_attention(dt, H, G, d, 2, 1, 16, [2500, 37], ws=ws)
    run_attention(dt, H, G, d, 2, 1, 16, [2500, 37], ws=ws, max_len=200)


def test_lengths_past_the_table_end_there():
    dims = dims_of(4, 4, 128, BF)
    kp, vp = pools(64, 512, BF)
    cache = A.PagedCache(kp.cuda(), vp.cuda(), 16, torch.tensor([[2, 0, 3]], dtype=torch.int32).cuda())
    q = torch.randn(1, 512).to(BF).cuda()
    a = A.acache_paged_attention(dims, cache, q, torch.tensor([48], dtype=torch.int32).cuda(), 1)
    b = A.acache_paged_attention(dims, cache, q, torch.tensor([2 ** 31 - 1], dtype=torch.int32).cuda(), 1)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dt,H,G,d", [SHAPES[1], SHAPES[3]])
def test_entries_that_name_no_block_read_as_zeros(dt, H, G, d):
    tables = torch.tensor([[3, -1, 1, 99], [0, 5, 2 ** 31 - 1, 4]], dtype=torch.int32)
    run_attention(dt, H, G, d, 2, 3, 16, [50, 64, 17, 64, 33, 60], tables=tables, kv=pools(10 * 16, G * d, dt), poison=False)


@pytest.mark.parametrize("dt,H,G,d", [SHAPES[0], SHAPES[1], SHAPES[3]])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_odd_numbers_reach_only_the_rows_that_attend(dt, H, G, d, bad):
    """A row that does not attend to a position is free of what K and V hold there, also beside one that does."""
    print(f"odd numbers {dt} {H}/{G} x {d}, {bad}", flush=True)
    per, n = 5, 70
    kp, vp = pools(8 * 16, G * d, dt, seed=21)
    tables = torch.tensor([[6, 2, 5, 0, 3]], dtype=torch.int32)
    lens = [60, 70, 61, 62, 3]
    vp[R.slot(tables, 8, 16, 0, 61), 1] = bad    # rows 1 and 3 see it
    vp[R.slot(tables, 8, 16, 0, 69), d - 1] = bad  # row 1
    vp[R.slot(tables, 8, 16, 0, 40)] = bad       # all but the last
    got, _ = run_attention(dt, H, G, d, 1, per, 16, lens, tables=tables, kv=(kp, vp), poison=False)
    assert torch.isfinite(got[4]).all() and not torch.isfinite(got[0]).any()
    kp, vp = pools(8 * 16, G * d, dt, seed=21)
    kp[R.slot(tables, 8, 16, 0, 65)] = math.nan   # row 1 alone
    got, lse = run_attention(dt, H, G, d, 1, per, 16, lens, tables=tables, kv=(kp, vp), poison=False)
    assert torch.isnan(got[1]).all() and torch.isfinite(got[[0, 2, 3, 4]]).all()


@pytest.mark.parametrize("dt,H,G,d", [SHAPES[0], SHAPES[3]])
def test_distant_logits(dt, H, G, d):
    """Maxima that rise far along the keys, in either order; a key whose logit is -inf; a row with nothing else."""
    kp, vp = pools(64 * 16, G * d, dt, seed=31)
    tables = some_tables(2, 30, 64)
    for p in range(300):
        kp[R.slot(tables, 64, 16, 0, p)] *= p / 20
        kp[R.slot(tables, 64, 16, 1, p)] *= (300 - p) / 20
    run_attention(dt, H, G, d, 2, 1, 16, [300, 300], tables=tables, kv=(kp, vp), poison=False)
    kp, vp = pools(64 * 16, G * d, dt, seed=32)
    q = torch.rand(2, H * d, generator=torch.Generator().manual_seed(1)).to(dt) + 0.5
    for p in (0, 7, 44):
        kp[R.slot(tables, 64, 16, 0, p)] = -math.inf
    for p in range(40):
        kp[R.slot(tables, 64, 16, 1, p)] = -math.inf
    got, lse = run_attention(dt, H, G, d, 2, 1, 16, [100, 40], tables=tables, kv=(kp, vp), poison=False, q=q)
    assert (got[1] == 0).all() and (lse[1] == -math.inf).all()


def test_shared_blocks_and_strided_pools():
    """Requests whose tables begin with the same blocks, pools with wider rows."""
    tables = torch.tensor([[4, 1, 7, 0], [4, 1, 2, 5], [4, 1, 7, 3]], dtype=torch.int32)
    run_attention(BF, 28, 4, 128, 3, 2, 16, [64, 63, 40, 41, 64, 50], tables=tables,
                  kv=pools(8 * 16, 4 * 128, BF, ld=4 * 128 + 8), poison=False)


def test_offsets_past_32_bits():
    """Slots whose element offsets pass 2^32, stored to and read from."""
    H = G = 32
    d, block = 128, 64
    n_blocks = 2 ** 32 // (G * d * block) + 40  # 4.3e9 elements and more
    dims = dims_of(H, G, d, BF)
    kd, vd = (torch.empty(n_blocks * block, G * d, dtype=BF, device="cuda") for _ in range(2))
    tables = torch.tensor([[n_blocks - 1, 1, n_blocks // 2 + 7, n_blocks - 30]], dtype=torch.int32)
    small = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32)
    ks, vs = (torch.zeros(4 * block, G * d, dtype=BF, device="cuda") for _ in range(2))
    x = torch.randn(250, 3 * G * d, device="cuda").to(BF)
    pos = torch.arange(250, dtype=torch.int32, device="cuda")
    lens = torch.full((250,), 250, dtype=torch.int32, device="cuda")
    res = []
    for kp, vp, t in ((kd, vd, tables), (ks, vs, small)):
        cache = A.PagedCache(kp, vp, block, t.cuda())
        q, k, v = x.split(G * d, 1)
        q = A.acache_paged_append(dims, cache, k, v, pos, 250, q=q)
        res.append((q, A.acache_paged_attention(dims, cache, q, lens, 250)))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    ref = R.attention(res[1][0][:2].cpu(), lens[:2].cpu(), ks.cpu(), vs.cpu(), block, small, H, G, d, 2)
    check(res[0][1][:2], ref[0], ref[2], "out")


def test_long_context():
    """One token over 200,000 positions of one KV head: many splits, values constant in V give themselves back."""
    dims = dims_of(1, 1, 128, BF)
    n, block = 200_003, 32
    n_blocks = -(-n // block)
    kp = torch.randn(n_blocks * block, 128, device="cuda").to(BF)
    vp = torch.ones_like(kp) * torch.arange(128, device="cuda").to(BF)
    t = torch.randperm(n_blocks, device="cuda").to(torch.int32)[None]
    cache = A.PagedCache(kp, vp, block, t)
    q = torch.randn(1, 128, device="cuda").to(BF)
    lse = torch.empty(1, 1, device="cuda")
    ws = A.paged_workspace(dims, cache, 1)
    assert A.acache_paged_attention_schedule(dims, cache, 1, 0, ws.nbytes) > 8
    out = A.acache_paged_attention(dims, cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), 1, lse=lse, ws=ws)
    want = torch.arange(128, dtype=torch.float64)
    # the weights' sum as rounded to bf16 against their own: half a step, and the result's rounding
    check(out, want[None], want[None] * (2.0 ** -8 * 2 + 1e-4), "out")
    slots = (t.long()[0][:, None] * block + torch.arange(block, device="cuda")).view(-1)[:n]
    logit = kp.double()[slots] @ q[0].double() / math.sqrt(128)
    assert abs(float(lse) - float(torch.logsumexp(logit, 0))) < 1e-3


def test_nothing_to_do():
    dims = dims_of(4, 4, 128, BF)
    kp, vp = (t.cuda() for t in pools(32, 512, BF))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rows = torch.empty(0, 512, dtype=BF, device="cuda")
    before = kp.clone()
    for batch, per in ((0, 3), (3, 0)):
        cache = A.PagedCache(kp, vp, 16, torch.zeros(batch, 2, dtype=torch.int32, device="cuda"))
        assert A.acache_paged_append(dims, cache, rows, rows, none, per, q=rows).shape == (0, 512)
        assert A.acache_paged_attention(dims, cache, rows, none, per).shape == (0, 512)
    cache = A.PagedCache(kp, vp, 16, torch.zeros(2, 0, dtype=torch.int32, device="cuda"))  # tables without entries
    q = torch.ones(2, 512, dtype=BF, device="cuda")
    A.acache_paged_append(dims, cache, q, q, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1)
    out = A.acache_paged_attention(dims, cache, q, torch.tensor([5, 1], dtype=torch.int32, device="cuda"), 1)
    assert (out == 0).all() and torch.equal(kp, before)
