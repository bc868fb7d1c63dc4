"""The 8-bit KV cache on the host: the reference's number format against
torch's, its store's rules on small cases, and the refusals of the entry
points (nothing is enqueued: the pointers are bogus).  CPU only."""

import ctypes

import numpy as np
import pytest
import torch

from tests import quant_reference as Q


@pytest.fixture(scope="module")
def A():
    from paper_2608_26140_amd import acache
    return acache


def test_table_and_rounding_match_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(Q.TABLE, codes.view(torch.float8_e4m3fn).double().numpy())
    rng = np.random.default_rng(3)
    y = np.concatenate([rng.normal(0, 1, 4000), rng.normal(0, 100, 4000).clip(-448, 448), rng.normal(0, 2e-3, 4000),
                        Q._MID, -Q._MID, Q._POS, -Q._POS]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(Q.encode(y.astype(np.float64)), want)


def test_exponent_is_the_smallest_that_fits():
    for amax in (0.0, 1e-38, 2.0 ** -108 * 1.75, 0.9, 1.0, 448.0, 448.0001, 447.9, 3.3e38, 1.75 * 2.0 ** 127):
        e = Q.exponent(amax)
        assert -117 <= e <= 119
        assert amax <= 448.0 * 2.0 ** e or e == 119
        assert e == -117 or amax > 448.0 * 2.0 ** (e - 1)


def test_store_rules():
    c = Q.Cache(np.full((10, 1, 16), 0xFF, np.uint8), np.zeros((3, 1)), 4)
    x = np.ones((2, 1, 16))
    c.store(x, [0, 1])                      # empty block, in part: the others become zeros
    assert c.scales[0, 0] == 2.0 ** -8 and c.codes[2, 0, 0] == 0 and c.values([0, 2])[:, 0, 0].tolist() == [1.0, 0.0]
    c.store(100 * x[:1], [2])               # a larger entry raises the scale, the others are rounded to it
    assert c.scales[0, 0] == 2.0 ** -2 and c.values([0, 2])[:, 0, 0].tolist() == [1.0, 96.0]
    c.store(0.01 * x, [0, 1])               # smaller entries leave it
    assert c.scales[0, 0] == 2.0 ** -2
    c.store(np.ones((4, 1, 16)), [0, 1, 2, 3])  # the whole block: the scale of its new rows
    assert c.scales[0, 0] == 2.0 ** -8
    c.store(np.ones((2, 1, 16)), [8, 9])    # the last, short block is whole
    assert c.scales[2, 0] == 2.0 ** -8 and c.scales[1, 0] == 0.0
    c.store(np.stack([3 * x[0], x[0]]), [8, 8])  # the last of equal slots
    assert c.values([8])[0, 0, 0] == 1.0 and np.isclose(c.values([9])[0, 0, 0], 1.0)


def pool(A, **kw):
    d = dict(k_codes=16, v_codes=16, k_scales=16, v_scales=16, ld=4096, n_slots=1000, block=64)
    d.update(kw)
    return A.QuantPoolDesc(**d)


def test_struct_layout(A):
    """As a C compiler lays acache_quant_pool out: four pointers, two int64, an int32, padded to 8."""
    offsets = [getattr(A.QuantPoolDesc, f).offset for f, _ in A.QuantPoolDesc._fields_]
    assert offsets == [0, 8, 16, 24, 32, 40, 48] and ctypes.sizeof(A.QuantPoolDesc) == 56


DIMS = (4096, 32, 32, 128, 12288, "bf16")


@pytest.mark.parametrize("kw,want", [
    (dict(k_codes=None), 1), (dict(v_codes=None), 1), (dict(k_scales=None), 1), (dict(v_scales=None), 1),
    (dict(ld=4095), 2), (dict(n_slots=-1), 2), (dict(n_slots=1 << 31), 2),
    (dict(block=0), 4), (dict(block=48), 4), (dict(block=8), 4), (dict(block=512), 4), (dict(block=-64), 4),
    (dict(ld=4104), 3), (dict(k_codes=24), 3), (dict(v_codes=8), 3),
])
def test_every_call_refuses_a_bad_pool(A, kw, want):
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)
    d = ctypes.byref(dims)
    bad = ctypes.byref(pool(A, **kw))
    assert lib.acache_quant_store(d, bad, p, p, 4096, 3, p, p, 1 << 30, None) == want
    assert lib.acache_quant_load(d, bad, p, 3, p, p, 4096, None) == want
    rg, keep = A._ragged([0, 3], [0, 5])
    assert lib.acache_quant_attention(d, ctypes.byref(rg), p, p, bad, p, None, None, 0, None) == want


def test_store_refusals(A):
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)
    good = pool(A)

    def call(dims=dims, pool=good, k=p, v=p, ld=4096, n=3, slots=p, ws=p, wsb=1 << 30):
        return lib.acache_quant_store(ctypes.byref(dims), None if pool is None else ctypes.byref(pool), k, v, ld, n,
                                      slots, ws, wsb, None)
    assert call(pool=None) == 1
    assert call(n=0, k=None, v=None, slots=None, ws=None) == 0
    assert call(n=-1) == 2
    assert call(k=None) == 1 and call(v=None) == 1 and call(slots=None) == 1
    assert call(ld=4088) == 2 and call(ld=4100) == 3
    assert call(k=ctypes.c_void_p(8)) == 3
    assert call(ws=None) == 5 and call(wsb=1000 * 4) == 5
    assert call(ws=ctypes.c_void_p(18)) == 5
    assert call(dims=A.make_dims(256, 4, 4, 40, 688, "f32")) == 4  # head_dim not a multiple of 16
    assert call(dims=A.make_dims(4096, 32, 32, 64, 12288, "bf16")) == 4


def test_load_refusals(A):
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)

    def call(k=p, v=p, ld=4096, n=3, slots=p):
        return lib.acache_quant_load(ctypes.byref(dims), ctypes.byref(pool(A)), slots, n, k, v, ld, None)
    assert call(n=0) == 0 and call(k=None, v=None) == 0
    assert call(n=-2) == 2 and call(slots=None) == 1 and call(ld=4000) == 2 and call(ld=4100) == 3
    assert call(v=ctypes.c_void_p(4)) == 3


def test_attention_refusals(A):
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)

    def call(dims=dims, rows=(0, 3), keys=(0, 5), q=p, slots=p, out=p, ws=None, wsb=0, desc=None):
        rg, keep = A._ragged(rows, keys)
        return lib.acache_quant_attention(ctypes.byref(dims), ctypes.byref(rg), q, slots,
                                          ctypes.byref(desc or pool(A)), out, None, ws, wsb, None)
    assert call(dims=A.make_dims(256, 4, 4, 64, 688, "f32")) == 4
    assert call(keys=(0, 0)) == 2            # rows without keys
    assert call(rows=(0, 0)) == 0            # no rows
    assert call(rows=(0, -1)) == 2 and call(rows=(1, 2)) == 2
    assert call(rows=tuple(range(66)), keys=tuple(range(66))) == 2  # batch above 64
    assert call(q=None) == 1 and call(slots=None) == 1 and call(out=None) == 1
    assert call(q=ctypes.c_void_p(8)) == 3 and call(out=ctypes.c_void_p(8)) == 3
    assert call(ws=ctypes.c_void_p(8), wsb=1 << 20) == 3
    assert call(desc=pool(A, n_slots=1 << 20)) == 4  # 2^20 rows of 4096 bytes: past 32-bit offsets


def test_sizes_past_a_launch_are_refused(A):
    """A launch holds fewer than 2^32 threads, a request's slots lie within 32-bit byte offsets."""
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)
    d = ctypes.byref(dims)
    big = 1 << 40

    def store(n, block):
        return lib.acache_quant_store(d, ctypes.byref(pool(A, block=block)), p, p, 4096, n, p, None, big, None)
    assert store(1 << 22, 16) == 4 and store((1 << 22) - 17, 16) == 5  # 5: the missing workspace, checked next
    assert store((1 << 26) - 300, 256) == 5 and store(1 << 26, 256) == 4

    def attend(rows, keys):
        rg, keep = A._ragged(rows, keys)
        return lib.acache_quant_attention(d, ctypes.byref(rg), p, p, ctypes.byref(pool(A)), p, None, ctypes.c_void_p(8),
                                          0, None)
    assert attend((0, 1 << 23), (0, 5)) == 3 and attend((0, (1 << 23) + 1), (0, 5)) == 4  # 3: the workspace's alignment
    assert attend((0, 1, 2), (0, 5, 5 + (1 << 29))) == 3 and attend((0, 1, 2), (0, 5, 6 + (1 << 29))) == 4
    assert attend((0, 1), (0, (1 << 31) - 1)) == 4

    def layer(rows, keys):
        rg, keep = A._ragged(rows, keys)
        lw = A.LayerWeights(*[16] * len(A.LayerWeights._fields_))
        return lib.acache_quant_layer_recompute(d, ctypes.byref(lw), ctypes.byref(rg), p, p, p, p, ctypes.byref(pool(A)),
                                                None, None, 0, None)
    assert layer((0, 3), (0, 1 << 29)) == 5 and layer((0, 3), (0, (1 << 29) + 1)) == 4


def test_workspace_size(A):
    lib, dims = A.lib, A.make_dims(*DIMS)

    def size(rows, **kw):
        return lib.acache_quant_workspace_size(ctypes.byref(dims), rows, ctypes.byref(pool(A, **kw)))
    assert size(0) >= 4 * (1000 + 16)
    assert size(0, n_slots=0) > 0            # 0 means refused
    sizes = [size(r) for r in (0, 1, 2, 32, 33, 300, 5000, 70000)]
    assert sizes == sorted(sizes)            # one workspace serves every smaller call
    assert size(-1) == 0 and size(1, block=48) == 0 and size(1, ld=64) == 0


def test_binding_refuses_before_the_call(A):
    dims = A.make_dims(256, 4, 2, 64, 688, "f32")
    c, s = torch.zeros(100, 128, dtype=torch.uint8), torch.zeros(7, 2)
    ok = A.QuantPool(c, c.clone(), s, s.clone(), 16)
    with pytest.raises(TypeError):
        A.QuantPool(c.float(), c, s, s, 16)
    with pytest.raises(ValueError):
        A.QuantPool(c, c[:50], s, s, 16)
    with pytest.raises(ValueError):
        A.QuantPool(c, c, s[:6], s[:6], 16)
    with pytest.raises(TypeError):
        A.QuantPool(c, c, s.double(), s.double(), 16)
    rows, slots = torch.zeros(3, 128), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):  # host tensors
        A.acache_quant_store(dims, ok, rows, rows, slots)
    with pytest.raises(TypeError):
        A.acache_quant_load(dims, ok, slots)
    with pytest.raises(TypeError):
        A.acache_quant_attention(dims, [0, 3], [0, 3], rows, slots, ok)


def test_clear_takes_whole_blocks(A):
    c = torch.zeros(100, 32, dtype=torch.uint8)
    p = A.QuantPool(c, c.clone(), torch.ones(7, 2), torch.ones(7, 2), 16)
    p.clear(slice(10, 50))                   # blocks 1 and 2 lie within
    assert p.k_scales[:, 0].tolist() == [1, 0, 0, 1, 1, 1, 1]
    p.clear(slice(90, 100))                  # the last block is 4 slots long
    assert p.v_scales[:, 1].tolist() == [1, 0, 0, 1, 1, 1, 0]
    p.clear(slice(50, 50))
    assert p.v_scales[:, 1].tolist() == [1, 0, 0, 1, 1, 1, 0]
    p.clear()
    assert not p.k_scales.any() and not p.v_scales.any()


def test_layer_refusals(A):
    lib, dims, p = A.lib, A.make_dims(*DIMS), ctypes.c_void_p(16)
    w = A.LayerWeights(16, 16, 16, 16, 16, 16)

    def call(dims=dims, rows=(0, 3), keys=(0, 5), x=p, pos=p, wsl=p, rsl=p, desc=None, ws=p, wsb=1 << 40, score=None):
        rg, keep = A._ragged(rows, keys)
        return lib.acache_quant_layer_recompute(
            ctypes.byref(dims), ctypes.byref(w), ctypes.byref(rg), x, pos, wsl, rsl, ctypes.byref(desc or pool(A)),
            ctypes.byref(score) if score else None, ws, wsb, None)
    assert call(dims=A.make_dims(256, 4, 4, 64, 688, "f32")) == 4
    assert call(rows=(0, 0)) == 0
    assert call(keys=(0, 0)) == 2
    assert call(x=None) == 1 and call(pos=None) == 1 and call(wsl=None) == 1 and call(rsl=None) == 1
    assert call(desc=pool(A, n_slots=0)) == 2
    assert call(desc=pool(A, n_slots=1 << 20)) == 4
    assert call(desc=pool(A, v_scales=None)) == 1 and call(desc=pool(A, block=24)) == 4
    assert call(x=ctypes.c_void_p(8)) == 3
    assert call(ws=None) == 5 and call(wsb=1000) == 5
    cq = (ctypes.c_int32 * 2)(0, 4)
    assert call(score=A.ScoreArgs(16, cq, 16, 10, 0, 16)) == 2      # more masked rows than rows
    cq2 = (ctypes.c_int32 * 2)(0, 2)
    assert call(score=A.ScoreArgs(16, cq2, 16, 10, 9, 16)) == 4     # unknown normalisation
    assert call(score=A.ScoreArgs(None, cq2, 16, 10, 0, 16)) == 1


def test_layer_workspace_size(A):
    lib, dims = A.lib, A.make_dims(*DIMS)

    def size(rows, batch=1, L=0, **kw):
        return lib.acache_quant_layer_workspace_size(ctypes.byref(dims), rows, batch, L, ctypes.byref(pool(A, **kw)))
    assert size(32) > lib.acache_workspace_size(ctypes.byref(dims), 32, 1, 0)
    assert size(700, 2, 512) >= size(700, 2, 100) >= size(700, 1, 100) >= size(600, 1, 100) > 0
    assert size(-1) == 0 and size(1, block=5) == 0
    f32 = A.make_dims(256, 4, 4, 64, 688, "f32")
    assert lib.acache_quant_layer_workspace_size(ctypes.byref(f32), 1, 1, 0, ctypes.byref(pool(A))) == 0
