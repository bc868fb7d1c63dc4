"""Which kernels the attention over an 8-bit cache launches: host arithmetic,
checked here so that a change of an estimate cannot take a way out of what the
GPU tests run.  CPU only."""

import ctypes

import pytest

from paper_2608_26140_amd import acache as A
from tests.quant_attention_cases import WAYS, cu, way_of


def partials(pairs):
    """What acache_quant_workspace_size gives for so many (row, head) pairs."""
    return min(65536, 64 * pairs) * 130 * 4


@pytest.mark.parametrize("way", WAYS)
def test_every_way_has_its_batch(way):
    _, H, Hkv, rows, keys, ws = WAYS[way]
    dims = A.make_dims(H * 128, H, Hkv, 128, 256, "bf16")
    pool = A.QuantPoolDesc(16, 16, 16, 16, Hkv * 128, 1900, 64)
    size = A.lib.acache_quant_workspace_size(ctypes.byref(dims), sum(rows), ctypes.byref(pool))
    assert size >= partials(sum(rows) * H)
    assert way_of(dims, rows, keys, size if ws else 0) == way


def test_tiles_cover_every_query():
    for H, Hkv, rows in ((4, 4, [1, 255, 256, 257]), (28, 4, [36, 37, 700]), (32, 32, [1089, 0, 654, 300])):
        dims = A.make_dims(H * 128, H, Hkv, 128, 256, "bf16")
        for S in (1, 64, 300, 5000):
            n = [r * (H // Hkv) for r in rows]
            wide, narrow, rest, splits = A.acache_quant_attention_schedule(dims, cu(rows), cu([S] * len(rows)), 0)
            assert splits == 1
            if wide and narrow:
                left = [x % 256 for x in n]
                assert wide == sum(x // 256 + (y > rest) for x, y in zip(n, left))
                assert narrow == sum(-(-y // 32) for y in left if y <= rest)
            else:
                assert (wide, narrow) in ((sum(-(-x // 256) for x in n), 0), (0, sum(-(-x // 32) for x in n)))


def test_splits_fit_the_workspace():
    dims = A.make_dims(4096, 32, 32, 128, 256, "bf16")
    most = A.acache_quant_attention_schedule(dims, [0, 32], [0, 8000], partials(32 * 32))[3]
    assert most > 4
    for s in range(1, most + 1):
        size = s * 32 * 32 * 130 * 4
        assert A.acache_quant_attention_schedule(dims, [0, 32], [0, 8000], size)[3] <= s
        assert A.acache_quant_attention_schedule(dims, [0, 32], [0, 8000], size - 1)[3] <= max(1, s - 1)


def test_refusals():
    dims = A.make_dims(4096, 32, 32, 128, 256, "bf16")
    out = [ctypes.c_int32(7) for _ in range(4)]

    def call(dims=dims, rows=(0, 3), keys=(0, 5), out=out):
        rg, keep = A._ragged(rows, keys)
        return A.lib.acache_quant_attention_schedule(ctypes.byref(dims), ctypes.byref(rg), 0,
                                                     *(o and ctypes.byref(o) for o in out))
    assert call(dims=A.make_dims(256, 4, 4, 64, 688, "f32")) == 4
    assert call(dims=A.make_dims(4096, 32, 32, 64, 256, "bf16")) == 4
    assert call(keys=(0, 0)) == 2 and call(rows=(1, 2)) == 2
    assert call(rows=(0, (1 << 23) + 1)) == 4 and call(keys=(0, (1 << 29) + 1)) == 4
    for i in range(4):
        assert call(out=[None if j == i else o for j, o in enumerate(out)]) == 1
    assert [o.value for o in out] == [7] * 4
    assert call(rows=(0, 0)) == 0 and [o.value for o in out] == [0, 0, 0, 1]
