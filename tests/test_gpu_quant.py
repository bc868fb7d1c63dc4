"""The 8-bit KV cache on the GPU against its float64 definition.  Stores and
loads are compared code for code.

Attention's bounds, for each output element o = sum_j p_j v_j (the cache's
values are exact in bf16, so only the arithmetic counts):
  * the output is rounded to bf16, and each weight is, before its product
    with V: half a step of bf16, 2^-8, of |o| and of sum_j p_j |v_j|;
  * a logit is a sum of 128 products in fp32 and is scaled and moved in fp32:
    132 roundings of 2^-24 of sum_i |q_i k_i| / sqrt(d); a weight is off by
    that much relatively, and so is the sum of the weights;
  * the weights' sum and the accumulation over S keys in fp32: S roundings.
The logarithm of the sum has the latter two, and the rounding of its own
last steps."""

import numpy as np
import pytest
import torch

from paper_2608_26140_amd import acache as A
from paper_2608_26140_amd import driver as D
from tests import quant_reference as Q
from tests.gpu_util import up_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"


def dims_of(dtype, H, Hkv, d):
    return A.make_dims(H * d, H, Hkv, d, 256, dtype)


def rows_of(x, dtype):
    """float64 [n, heads, d] as device rows, and the same values in float64."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t.flatten(1).to(DEV), t.double().numpy()


class Pair:
    """A device cache and the reference's K and V, kept side by side."""

    def __init__(self, dtype, Hkv, d, n_slots, block, H=None, ld=None, seed=0):
        self.dims = dims_of(dtype, H or Hkv, Hkv, d)
        self.dtype, self.Hkv, self.d, self.n_slots, self.block = dtype, Hkv, d, n_slots, block
        rng = np.random.default_rng(seed)
        row = Hkv * d
        self.ld = ld or row
        # codes of an empty cache are arbitrary: NaN codes among them
        self.raw = [rng.integers(0, 256, (n_slots, self.ld), dtype=np.uint8) for _ in range(2)]
        dev = [torch.from_numpy(r).to(DEV) for r in self.raw]
        self.dev = dev
        n_blocks = -(-n_slots // block)
        sc = [torch.zeros(n_blocks, Hkv, device=DEV) for _ in range(2)]
        self.pool = A.QuantPool(dev[0][:, :row], dev[1][:, :row], sc[0], sc[1], block)
        self.ref = [Q.Cache(r[:, :row].reshape(n_slots, Hkv, d), np.zeros((n_blocks, Hkv)), block) for r in self.raw]
        self.ws = A.quant_workspace(self.dims, 0, self.pool)
        self.ws.fill_(0x5A)  # no initial contents are needed
        self.rng = rng

    def store(self, slots, spread=1.0, x=None, check=True, reference=True):
        n = len(slots)
        src = []
        for i in range(2):
            v = self.rng.normal(0, spread, (n, self.Hkv, self.d)) if x is None else x[i]
            t, v64 = rows_of(v, self.dtype)
            src.append(t)
            if reference:
                self.ref[i].store(v64, slots)
        A.acache_quant_store(self.dims, self.pool, *src, up_i32(slots), ws=self.ws)
        if check:
            self.check()

    def check(self):
        torch.cuda.synchronize()
        row = self.Hkv * self.d
        for i, (scales, name) in enumerate(((self.pool.k_scales, "K"), (self.pool.v_scales, "V"))):
            np.testing.assert_array_equal(scales.cpu().numpy().astype(np.float64), self.ref[i].scales, err_msg=f"{name} scales")
            got = self.dev[i].cpu().numpy()
            np.testing.assert_array_equal(got[:, row:], self.raw[i][:, row:], err_msg=f"{name}: bytes beside the rows")
            g, r = got[:, :row].reshape(self.n_slots, self.Hkv, self.d), self.ref[i].codes
            nan = (g & 127) == 127
            np.testing.assert_array_equal(nan, (r & 127) == 127, err_msg=f"{name}: NaN codes")
            np.testing.assert_array_equal(np.where(nan, 0, g), np.where(nan, 0, r), err_msg=f"{name} codes")


SHAPES = [("bf16", 4, 128), ("bf16", 1, 128), ("f32", 2, 32), ("f32", 3, 48), ("f32", 4, 128), ("f32", 1, 16)]


@pytest.mark.parametrize("dtype,Hkv,d", SHAPES)
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
def test_store_sequence(dtype, Hkv, d, block):
    """Whole blocks, parts of blocks that grow, shrink or keep the scale, the
    short last block, one row, rows out of range and slots named twice."""
    n_slots = 3 * block + block // 2 + 1
    p = Pair(dtype, Hkv, d, n_slots, block, seed=block + d)
    p.store(np.arange(block))                          # one whole block
    p.store(np.arange(block - 3, block + 5), 0.1)      # the end of it and the start of an empty one
    p.store([5], 30.0)                                 # one larger row
    p.store(np.arange(7, 9), 1e-3)                     # smaller ones
    p.store(np.arange(3 * block, n_slots))             # the short last block
    p.store(p.rng.permutation(n_slots)[:2 * block], 3.0)
    p.store([-1, n_slots, 2 ** 31 - 1, -2 ** 31, 3], 2.0)
    p.store([9, 9, 4, 9, 4, block + 1, 4])             # equal slots: the last row
    p.store(np.arange(n_slots), 0.5)                   # everything


@pytest.mark.parametrize("n,n_slots", [(1, 1), (2, 5), (1000, 1100), (1024, 1024), (1025, 3000), (2500, 5003), (9000, 9001)])
@pytest.mark.parametrize("order", ["runs", "shuffled", "twice"])
def test_store_sizes(n, n_slots, order):
    p = Pair("bf16", 2, 128, n_slots, 64, seed=n)
    if order == "runs":
        slots = np.arange(n) + (n_slots - n) // 2
    elif order == "shuffled":
        slots = p.rng.permutation(n_slots)[:n]
    else:
        slots = p.rng.integers(-2, n_slots + 2, n)
    p.store(slots)
    p.store(slots[::-1].copy(), 4.0)


@pytest.mark.parametrize("n", [200, 1500])
def test_store_rows_past_the_short_last_block(n):
    """Rows whose slot is not there, with numbers in the short last block's
    range, behind and between the last rows of that block."""
    n_slots = 32 * 64 + 20
    p = Pair("bf16", 2, 128, n_slots, 64, seed=n)
    slots = np.arange(n_slots - n, n_slots)
    p.store(np.concatenate([slots, [n_slots, n_slots + 43]]))
    p.store(np.concatenate([slots[:-5], [n_slots + 1], slots[-5:], [n_slots + 2, -1]]), 3.0)
    p.store(np.concatenate([[n_slots], slots[::-1], [n_slots - 3, n_slots + 7, n_slots - 1, n_slots]]), 0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_special_values(dtype):
    d = 128
    vals = [0.0, -0.0, np.inf, -np.inf, np.nan, 448.0, -448.0, 464.0, 1e-30, -1e-38, 1e-45, 3.3e38, -3.3e38, 1.75 * 2.0 ** 127,
            2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 1.0625, 1.1875]
    for k, v in enumerate(vals):
        p = Pair(dtype, 1, d, 40, 16, seed=k)
        x = np.zeros((16, 1, d))
        x[3, 0, 5] = v
        x[4, 0, 6] = 1e-3 * (k % 2)
        with np.errstate(over="ignore", invalid="ignore"):
            p.store(np.arange(16), x=[x, -x])
            p.store(np.arange(20, 25), x=[np.full((5, 1, d), v), x[:5]])
            p.store([21], x=[np.full((1, 1, d), 7.0), np.full((1, 1, d), v)])


def test_store_all_codes_and_ties():
    """Every e4m3 value, the midpoints between them and their neighbours."""
    pos = Q._POS
    y = np.concatenate([pos, Q._MID, np.nextafter(Q._MID.astype(np.float32), np.float32(0)),
                        np.nextafter(Q._MID.astype(np.float32), np.float32(1e9)), [448.0] * 4])
    y = np.concatenate([y, -y])
    n = -(-y.size // 128)
    x = np.zeros((n + 1, 1, 128))
    x.reshape(-1)[:y.size] = y
    x[-1] = 448.0
    for scale in (1.0, 2.0 ** -117, 2.0 ** 100):
        p = Pair("f32", 1, 128, 32, 16)
        p.store(np.arange(n + 1), x=[x * scale, x[::-1] * scale])


def test_store_strided_rows_and_pool():
    """Rows that are columns of a wider product, and a pool whose rows are
    wider than the heads: what lies beside them stays."""
    p = Pair("bf16", 2, 128, 200, 64, ld=2 * 128 + 48, seed=1)
    p.store(np.arange(30, 130))
    n = 77
    wide = torch.randn(n, 1024, device=DEV).to(torch.bfloat16)
    k, v = wide[:, 256:512], wide[:, 768:]
    slots = p.rng.permutation(200)[:n]
    for i, t in enumerate((k, v)):
        p.ref[i].store(t.double().cpu().numpy().reshape(n, 2, 128), slots)
    A.acache_quant_store(p.dims, p.pool, k, v, up_i32(slots), ws=p.ws)
    p.check()


def test_clear_empties():
    p = Pair("bf16", 2, 128, 200, 64, seed=2)
    p.store(np.arange(200), 50.0)
    p.pool.clear(slice(64, 128))
    for r in p.ref:
        r.scales[1] = 0.0
    k, _ = A.acache_quant_load(p.dims, p.pool, up_i32([63, 64, 127, 128]))
    assert not k[1:3].any() and k[0].any() and k[3].any()
    p.store([70, 100], 1.0)  # the scale of the new rows, zeros beside them


@pytest.mark.parametrize("dtype,Hkv,d", SHAPES)
def test_load(dtype, Hkv, d):
    p = Pair(dtype, Hkv, d, 333, 32, seed=d)
    x = p.rng.normal(0, 2, (250, Hkv, d))
    x[7] = np.nan
    p.store(np.arange(250), x=[x, 3 * x])
    p.store(np.arange(250, 260), 1e-36, check=False)
    for slots in ([0], [332], np.arange(333), p.rng.integers(-3, 340, 1001), [-1, 333, 2 ** 31 - 1, -2 ** 31]):
        k, v = A.acache_quant_load(p.dims, p.pool, up_i32(slots))
        for got, ref in ((k, p.ref[0]), (v, p.ref[1])):
            np.testing.assert_array_equal(got.double().cpu().numpy().reshape(len(slots), Hkv, d), ref.values(slots))


def test_load_one_of_two_and_strided():
    p = Pair("bf16", 2, 128, 100, 16, seed=4)
    p.store(np.arange(90))
    slots = p.rng.permutation(100)[:41]
    wide = torch.full((41, 1024), 3.0, dtype=torch.bfloat16, device=DEV)
    k, v = A.acache_quant_load(p.dims, p.pool, up_i32(slots), v_out=wide[:, 512:768])
    assert k is None
    np.testing.assert_array_equal(v.double().cpu().numpy().reshape(41, 2, 128), p.ref[1].values(slots))
    assert (wide[:, :512] == 3).all() and (wide[:, 768:] == 3).all()


def test_stream_of_workspace_and_results():
    """What a call on another stream makes for itself is that stream's: neither
    its workspace nor its results use memory that the current stream still
    works with, and the workspace is not given away before the call has run."""
    p = Pair("bf16", 2, 128, 4000, 64, seed=6)
    slots = p.rng.permutation(4000)[:3000]
    x = [p.rng.normal(0, 1, (3000, 2, 128)) for _ in range(2)]
    src = [rows_of(v, "bf16") for v in x]
    dst = up_i32(slots)
    for r, (_, v64) in zip(p.ref, src):
        r.store(v64, slots)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    A.acache_quant_store(p.dims, p.pool, src[0][0], src[1][0], dst, stream=other)
    scrap = [torch.full((5000,), 7, dtype=torch.int32, device=DEV) for _ in range(8)]  # the current stream's
    k, v = A.acache_quant_load(p.dims, p.pool, dst, stream=other)
    q = torch.randn(40, 256, device=DEV).to(torch.bfloat16)
    torch.cuda.current_stream().synchronize()
    lse = torch.empty(40, 2, device=DEV)
    out = A.acache_quant_attention(p.dims, [0, 40], [0, 3000], q, dst, p.pool, lse=lse, stream=other)
    torch.cuda.synchronize()
    p.check()
    for got, ref in ((k, p.ref[0]), (v, p.ref[1])):
        np.testing.assert_array_equal(got.double().cpu().numpy().reshape(3000, 2, 128), ref.values(slots))
    check_attention(p, q, [0, 40], [0, 3000], slots, out, lse, "another stream")
    assert all((t == 7).all() for t in scrap)


# ---------------------------------------------------------------------------- attention
def check_attention(p, q, cu_rows, cu_keys, slots, out, lse, what=""):
    H, Hkv, d = p.dims.n_heads, p.Hkv, p.d
    out, lse = out.double().cpu().numpy().reshape(-1, H, d), lse.double().cpu().numpy()
    q64 = q.double().cpu().numpy().reshape(-1, H, d)
    for b in range(len(cu_rows) - 1):
        r0, r1 = cu_rows[b], cu_rows[b + 1]
        if r0 == r1:
            continue
        sl = slots[cu_keys[b]:cu_keys[b + 1]]
        ref, ref_lse, weight, big = Q.attention(q64[r0:r1], p.ref[0].values(sl), p.ref[1].values(sl), H // Hkv)
        logit = 132 * 2.0 ** -24 * big
        total = logit + (len(sl) + 8) * 2.0 ** -24
        bound = 2.0 ** -8 * (np.abs(ref) + weight) * 1.01 + (2 * total)[..., None] * weight + 1e-30
        err = np.abs(out[r0:r1] - ref)
        worst = float((err / bound).max())
        print(f"[attention] {what} request {b}: {worst:.3f} of the bound, lse {np.abs(lse[r0:r1] - ref_lse).max():.2e}", flush=True)
        assert np.all(np.isfinite(out[r0:r1])) and worst <= 1.0
        assert np.all(np.abs(lse[r0:r1] - ref_lse) <= total + 2.0 ** -21 * (1 + np.abs(ref_lse)))


def run_attention(p, rows, keys, slots, q=None, ws=True, what="", poison=True):
    cu_rows = np.concatenate([[0], np.cumsum(rows)]).astype(int).tolist()
    cu_keys = np.concatenate([[0], np.cumsum(keys)]).astype(int).tolist()
    H, d = p.dims.n_heads, p.d
    n = cu_rows[-1]
    if q is None:
        q = torch.from_numpy(p.rng.normal(0, 1.3, (n, H * d))).to(torch.bfloat16).to(DEV)
    out = torch.full((n + 1, H * d), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n + 1, H), float("nan"), device=DEV)
    w = None
    if ws:
        w = A.quant_workspace(p.dims, n, p.pool)
        w.fill_(0xFF)  # NaN partials
    A.acache_quant_attention(p.dims, cu_rows, cu_keys, q, up_i32(slots), p.pool, out=out, lse=lse, ws=w)
    torch.cuda.synchronize()
    assert torch.isnan(out[n]).all() and torch.isnan(lse[n]).all()  # what lies behind the rows stays
    check_attention(p, q, cu_rows, cu_keys, slots, out[:n], lse[:n], what)
    return out[:n], lse[:n]


HEADS = [(4, 4), (28, 4), (8, 1), (4, 2), (3, 3)]


def filled(H, Hkv, n_slots, block, seed=0, spread=True):
    p = Pair("bf16", Hkv, 128, n_slots, block, H=H, seed=seed)
    x = [p.rng.normal(0, 1.3, (n_slots, Hkv, 128)) for _ in range(2)]
    if spread:  # blocks of unequal scales
        for v in x:
            v *= 2.0 ** p.rng.integers(-3, 2, (n_slots // 16 + 1, Hkv)).repeat(16, 0)[:n_slots, :, None]
    p.store(np.arange(n_slots), x=x, check=False)
    return p


@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 65, 130, 257])
def test_attention_rows_and_heads(H, Hkv, rows):
    p = filled(H, Hkv, 700, 64, seed=rows)
    for S in (1, 63, 500):
        slots = p.rng.integers(0, 700, S)
        run_attention(p, [rows], [S], slots, what=f"{H}/{Hkv} {rows} x {S}")


@pytest.mark.parametrize("S", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 191, 256, 1000, 2051])
@pytest.mark.parametrize("rows", [1, 40])
def test_attention_keys(S, rows):
    p = filled(4, 2, 2100, 32, seed=S)
    run_attention(p, [rows], [S], p.rng.permutation(2100)[:S], what=f"{rows} x {S}")


@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
def test_attention_blocks(block):
    p = filled(4, 2, 900, block, seed=block)
    run_attention(p, [40, 3], [777, 123], p.rng.integers(0, 900, 900), what=f"block {block}")


@pytest.mark.parametrize("ws", [True, False])
def test_attention_ragged(ws):
    """Requests without rows or with few, of unequal numbers of keys; a
    request without keys has no rows."""
    p = filled(8, 2, 1500, 64, seed=9)
    rows, keys = [5, 0, 300, 1, 0, 64, 31], [1400, 10, 3, 700, 0, 65, 1]
    run_attention(p, rows, keys, p.rng.integers(0, 1500, sum(keys)), ws=ws, what="ragged")


@pytest.mark.parametrize("H,Hkv,rows", [(4, 4, 1), (28, 4, 9), (4, 2, 600)])
def test_attention_absent_slots_and_empty_blocks(H, Hkv, rows):
    """Slots outside the cache and empty blocks are keys and values of zeros,
    whatever the codes; NaN in slots that are not read does not show."""
    p = filled(H, Hkv, 640, 64, seed=11)
    p.pool.clear(slice(128, 256))
    for r in p.ref:
        r.scales[2:4] = 0.0
    x = np.full((1, Hkv, 128), np.nan)
    p.store([300], x=[x, x], check=False)
    slots = p.rng.integers(-60, 700, 901)
    slots[slots == 300] = 301
    slots[:70] = -1
    slots[-5:] = [2 ** 31 - 1, -2 ** 31, 640, 0, -1]
    run_attention(p, [rows], [901], slots, what="absent")
    run_attention(p, [rows], [3], [-1, -5, 640], what="only absent")


@pytest.mark.parametrize("rows", [1, 33, 300])
def test_attention_large_logits(rows):
    """Logits of some hundreds, a key that dominates, maxima that move late."""
    p = filled(4, 2, 1000, 64, seed=12)
    q = torch.from_numpy(p.rng.normal(0, 60, (rows, 512))).to(torch.bfloat16).to(DEV)
    run_attention(p, [rows], [990], np.arange(990), q=q, what="large")
    big = np.zeros((1, 2, 128)) + 40.0
    p.store([999], x=[big, big], check=False)
    run_attention(p, [rows], [500], np.r_[np.arange(499), 999], what="last dominates")
    run_attention(p, [rows], [500], np.r_[999, np.arange(499)], what="first dominates")


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_attention_extreme_scales(rows):
    """Queries and keys whose elements span the types' ranges: rows of tiny
    queries, of one large element beside small ones, keys of the smallest and
    of large scales, and zero queries."""
    p = Pair("bf16", 2, 128, 320, 64, H=4, seed=13)
    x = p.rng.normal(0, 1, (320, 2, 128))
    x[:64] *= 1e-36
    x[64:128] *= 1e4
    x[128:192, :, 7] *= 300
    v = p.rng.normal(0, 1, (320, 2, 128))
    v[64:128] *= 1e-30
    p.store(np.arange(320), x=[x * 1e-4, v], check=False)
    q = p.rng.normal(0, 1, (rows, 512))
    q[0::5] *= 1e-3
    q[1::5, ::64] *= 1e4
    q[1::5] *= 1e-4
    q[2::5] = 0.0
    q[3::5] *= 1e-38
    q = torch.from_numpy(q).to(torch.bfloat16).to(DEV)
    run_attention(p, [rows], [320], np.arange(320), q=q, what="extreme")


def test_scales_are_read_as_powers_of_two():
    """Scales of any significand give the bits of the powers of two at or below
    them, in every reader and in a store that keeps entries."""
    p = filled(4, 4, 600, 32, seed=23)
    slots = up_i32(p.rng.permutation(600))
    q = [torch.randn(r, 512, device=DEV).to(torch.bfloat16) for r in (1, 64 * 256)]
    new = [torch.randn(9, 512, device=DEV).to(torch.bfloat16) for _ in range(2)]

    def read():
        one = A.acache_quant_attention(p.dims, [0, 1], [0, 600], q[0], slots, p.pool, ws=p.ws)
        many = A.acache_quant_attention(p.dims, np.arange(65) * 256, np.arange(65) * 9, q[1], slots, p.pool)
        return (one, many, *A.acache_quant_load(p.dims, p.pool, slots))

    def store():
        A.acache_quant_store(p.dims, p.pool, *new, slots[:9].contiguous(), ws=p.ws)
        return read()
    state = [t.clone() for t in (*p.dev, p.pool.k_scales, p.pool.v_scales)]
    want = read(), store()
    for t, was in zip((*p.dev, p.pool.k_scales, p.pool.v_scales), state):
        t.copy_(was)
    for t in (p.pool.k_scales, p.pool.v_scales):
        t.mul_(1.0 + 0.999 * torch.rand(t.shape, device=DEV))
    got = read(), store()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w, g))


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_attention_nan_shows(rows):
    """A NaN key makes every row that reads it NaN; other heads and requests stay."""
    p = filled(4, 2, 256, 64, seed=14)
    x = p.rng.normal(0, 1, (1, 2, 128))
    x[0, 1, 3] = np.nan
    p.store([100], x=[x, np.nan_to_num(x)], check=False)
    q = torch.from_numpy(p.rng.normal(0, 1, (2 * rows, 512))).to(torch.bfloat16).to(DEV)
    slots = up_i32(np.r_[np.arange(90, 200), np.arange(110, 200)])
    out = A.acache_quant_attention(p.dims, [0, rows, 2 * rows], [0, 110, 200], q, slots, p.pool,
                                   ws=A.quant_workspace(p.dims, 2 * rows, p.pool)).view(2, rows, 4, 128)
    assert torch.isnan(out[0, :, 2:]).all()
    assert torch.isfinite(out[0, :, :2]).all() and torch.isfinite(out[1]).all()


@pytest.mark.parametrize("rows", [1, 64, 300])
def test_attention_matches_bf16_attention_of_the_values_read_back(rows):
    """acache_attention on the pools read back is the same operation."""
    p = filled(8, 4, 1200, 64, seed=15)
    k, v = A.acache_quant_load(p.dims, p.pool, up_i32(np.arange(1200)))
    q = torch.from_numpy(p.rng.normal(0, 1.3, (2 * rows, 1024))).to(torch.bfloat16).to(DEV)
    slots = up_i32(p.rng.integers(0, 1200, 1100))
    cu = [0, rows, 2 * rows], [0, 1000, 1100]
    got = A.acache_quant_attention(p.dims, *cu, q, slots, p.pool, ws=A.quant_workspace(p.dims, 2 * rows, p.pool))
    ref = A.acache_attention(p.dims, *cu, q, slots, k, v)
    weight = A.acache_attention(p.dims, *cu, q, slots, k, v.abs()).double()
    # both round the weights and the output: twice the bound of each
    assert ((got.double() - ref.double()).abs() <= 2 * 2.0 ** -8 * (ref.double().abs() + 1.02 * weight) * 1.05).all()


def test_attention_strided_pool_and_other_stream():
    p = Pair("bf16", 2, 128, 300, 64, H=4, ld=320, seed=16)
    p.store(np.arange(300))
    side = torch.cuda.Stream()
    q = torch.randn(50, 512, device=DEV).to(torch.bfloat16)
    slots = p.rng.integers(0, 300, 290)
    ws = A.quant_workspace(p.dims, 50, p.pool)
    dev_slots = up_i32(slots)
    lse = torch.empty(50, 4, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    A.acache_quant_attention(p.dims, [0, 50], [0, 290], q, dev_slots, p.pool, out=out, lse=lse, ws=ws, stream=side)
    side.synchronize()
    check_attention(p, q, [0, 50], [0, 290], slots, out, lse, "strided")


def test_attention_near_the_offset_limit():
    """A pool of almost 2^31 bytes: slots at its end."""
    n_slots = (1 << 31) // 4096 - 1
    dims = dims_of("bf16", 4, 4, 128)
    kc, vc = (torch.empty(n_slots, 4096, dtype=torch.uint8, device=DEV) for _ in range(2))
    sc = [torch.zeros(-(-n_slots // 64), 4, device=DEV) for _ in range(2)]
    pool = A.QuantPool(kc, vc, *sc, 64)
    rng = np.random.default_rng(1)
    slots = n_slots - 1 - np.arange(200)
    x = [rows_of(rng.normal(0, 1, (200, 4, 128)), "bf16") for _ in range(2)]
    A.acache_quant_store(dims, pool, x[0][0], x[1][0], up_i32(slots))
    k, v = A.acache_quant_load(dims, pool, up_i32(slots))
    q = torch.randn(70, 512, device=DEV).to(torch.bfloat16)
    order = rng.permutation(200)
    out = A.acache_quant_attention(dims, [0, 70], [0, 200], q, up_i32(slots[order]), pool,
                                   ws=A.quant_workspace(dims, 70, pool))
    k64, v64 = (t.double().cpu().numpy().reshape(200, 4, 128)[order] for t in (k, v))
    ref, _, weight, big = Q.attention(q.double().cpu().numpy().reshape(70, 4, 128), k64, v64, 1)
    bound = 2.0 ** -8 * 1.01 * (np.abs(ref) + weight) + (2 * (132 * big + 208) * 2.0 ** -24)[..., None] * weight
    assert (np.abs(out.double().cpu().numpy().reshape(70, 4, 128) - ref) <= bound).all()
    assert np.abs(k64).max() > 1  # the rows arrived


# Many queries: the 256-query kernel (whole tiles, one of 64 requests each a
# workgroup a head; few keys up), with key splits, and with the 32-query kernel
# on what is left of the requests.
MANY = [
    ("one key", 4, 4, [256] * 64, [1] * 64),
    ("two tiles of keys and fewer", 4, 4, [256 - b % 5 * 7 for b in range(64)], [33 + b for b in range(64)]),
    ("ragged", 4, 4, [256 - b % 5 * 7 for b in range(64)], [500 - 3 * b for b in range(64)]),
    ("grouped heads", 28, 4, [36] * 64, [300 + b for b in range(64)]),
    ("some without rows", 4, 2, [0 if b % 9 == 4 else 500 for b in range(64)], [901 - b for b in range(64)]),
    ("key splits", 28, 4, [256, 200], [5120, 4999]),
    ("more key splits", 16, 4, [256, 300], [5000, 5063]),
    ("with remainders", 4, 4, [286 - b % 7 for b in range(64)], [600 - b for b in range(64)]),
    ("grouped, with remainders", 8, 1, [130] * 64, [900 - b for b in range(64)]),
    ("long and short remainders", 32, 32, [794 - 11 * b for b in range(8)], [2432 - 17 * b for b in range(8)]),
]


def sampled(cu_rows, per, rng):
    """A few rows of each request, its first and last among them."""
    return [np.unique(np.r_[a, b - 1, rng.integers(a, b, per)]) if b > a else np.zeros(0, dtype=int)
            for a, b in zip(cu_rows[:-1], cu_rows[1:])]


def check_many(p, rows, keys, slots, q, out, lse, what):
    cu_rows, cu_keys = (np.concatenate([[0], np.cumsum(n)]).astype(int) for n in (rows, keys))
    rows_of_req = sampled(cu_rows, 3, p.rng)
    at = torch.from_numpy(np.concatenate(rows_of_req)).to(DEV)
    cu = np.concatenate([[0], np.cumsum([len(r) for r in rows_of_req])]).astype(int).tolist()
    check_attention(p, q[at], cu, cu_keys.tolist(), slots, out[at], lse[at], what)


def many(p, rows, keys, slots, q=None, ws=True, what=""):
    n, H = int(np.sum(rows)), p.dims.n_heads
    cu_rows, cu_keys = (np.concatenate([[0], np.cumsum(x)]).astype(int).tolist() for x in (rows, keys))
    if q is None:
        q = (1.3 * torch.randn(n, H * 128, device=DEV, generator=torch.Generator(DEV).manual_seed(n))).to(torch.bfloat16)
    out = torch.full((n + 1, H * 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n + 1, H), float("nan"), device=DEV)
    w = None
    if ws:
        w = A.quant_workspace(p.dims, n, p.pool)
        w.fill_(0xFF)
    A.acache_quant_attention(p.dims, cu_rows, cu_keys, q, up_i32(slots), p.pool, out=out, lse=lse, ws=w)
    torch.cuda.synchronize()
    assert torch.isnan(out[n]).all() and torch.isnan(lse[n]).all()
    assert torch.isfinite(out[:n].float()).all() and torch.isfinite(lse[:n]).all()
    check_many(p, rows, keys, slots, q, out[:n], lse[:n], what)
    return out[:n], lse[:n]


@pytest.mark.parametrize("what,H,Hkv,rows,keys", MANY, ids=[m[0] for m in MANY])
def test_attention_many_queries(what, H, Hkv, rows, keys):
    p = filled(H, Hkv, 1900, 64, seed=len(what))
    p.pool.clear(slice(640, 768))  # two empty blocks
    for r in p.ref:
        r.scales[10:12] = 0.0
    slots = p.rng.integers(-40, 1940, int(np.sum(keys)))
    out, lse = many(p, rows, keys, slots, what=what)
    again, lse2 = many(p, rows, keys, slots, what=what + ", again")
    assert torch.equal(out, again) and torch.equal(lse, lse2)  # the same bits every time
    many(p, rows, keys, slots, ws=False, what=what + ", no workspace")


def test_attention_many_queries_values():
    """Logits of some hundreds, maxima that move late, NaN in one key."""
    p = filled(4, 4, 1000, 64, seed=31)
    rows, keys = [256] * 64, [300] * 64
    big = np.zeros((1, 4, 128)) + 40.0
    p.store([999], x=[big, big], check=False)
    slots = p.rng.integers(0, 999, 64 * 300).reshape(64, 300)
    slots[::2, -1] = 999
    slots[1::2, 0] = 999
    g = torch.Generator(DEV).manual_seed(5)
    q = (20 * torch.randn(64 * 256, 512, device=DEV, generator=g)).to(torch.bfloat16)
    many(p, rows, keys, slots.reshape(-1), q=q, what="large")
    x = p.rng.normal(0, 1, (1, 4, 128))
    x[0, 2, 3] = np.nan
    p.store([998], x=[x, np.nan_to_num(x)], check=False)
    slots[:, 150] = 997
    slots[slots == 998] = 996
    slots[5, 150] = 998
    out = A.acache_quant_attention(p.dims, np.arange(65) * 256, np.arange(65) * 300, q, up_i32(slots.reshape(-1)), p.pool)
    bad = torch.isnan(out.view(64, 256, 4, 128)).any(-1)
    assert bad[5, :, 2].all() and int(bad.sum()) == 256


# ---------------------------------------------------------------------------- together
def test_store_attend_load_together_and_captured():
    """A decode loop's calls: rows of a block overwrite their slots, the view
    made by acache_build_maps is attended to, rows are read back; captured
    into a graph and replayed, with eager calls on other data between the
    replays, each replay gives the eager calls' bits for the data it has."""
    B, L, own, k_anchor, rows = 3, 200, 80, 37, 16
    S, R = L + own, k_anchor + own
    lay = A.Layout(S, 0, L, S - 32, 32, 0, L, R)
    rng = np.random.default_rng(5)
    anchors = np.stack([np.sort(rng.permutation(L)[:k_anchor]) for _ in range(B)])
    m = A.acache_build_maps(lay, B, up_i32(anchors), k_anchor)
    p = Pair("bf16", 2, 128, L + B * R, 16, H=6, seed=17)
    p.store(np.arange(L + B * R))
    view = m["read_slots"].cpu().numpy()
    step_slots = np.concatenate([m["write_slots"].cpu().numpy()[b * R + R - 32:b * R + R - 32 + rows] for b in range(B)])
    dst = up_i32(step_slots)
    ks, vs = (torch.empty(B * rows, 256, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty(B * rows, 768, dtype=torch.bfloat16, device=DEV)
    ws = A.quant_workspace(p.dims, B * rows, p.pool)
    out = torch.empty_like(q)
    lse = torch.empty(B * rows, 6, device=DEV)
    back = [torch.empty_like(ks) for _ in range(2)]
    cu_rows, cu_keys = [b * rows for b in range(B + 1)], [b * S for b in range(B + 1)]

    def step():
        A.acache_quant_store(p.dims, p.pool, ks, vs, dst, ws=ws)
        A.acache_quant_attention(p.dims, cu_rows, cu_keys, q, m["read_slots"], p.pool, out=out, lse=lse, ws=ws)
        A.acache_quant_load(p.dims, p.pool, dst, *back)

    def new_data(spread):
        x = [rng.normal(0, spread, (B * rows, 2, 128)) for _ in range(2)]
        for t, v, r in zip((ks, vs), x, p.ref):
            rows_dev, v64 = rows_of(v, "bf16")
            t.copy_(rows_dev)
            r.store(v64, step_slots)
        q.copy_(torch.from_numpy(rng.normal(0, 1.3, (B * rows, 768))).to(torch.bfloat16))

    def check(what):
        torch.cuda.synchronize()
        p.check()
        check_attention(p, q, cu_rows, cu_keys, view, out, lse, what)
        for t, r in zip(back, p.ref):
            np.testing.assert_array_equal(t.double().cpu().numpy().reshape(-1, 2, 128), r.values(step_slots))

    new_data(1.0)
    step()
    check("eager")
    graph, _ = D.capture(step)
    for i, spread in enumerate((0.5, 40.0, 1.0, 3.0)):
        new_data(spread)
        graph.replay()
        check(f"replay {i}")
        kept = out.clone(), lse.clone(), p.pool.k_scales.clone()
        step()  # eager, the same data: the same bits
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, (out, lse, p.pool.k_scales)))
        new_data(0.7 * spread)
        step()
        check(f"eager after replay {i}")
