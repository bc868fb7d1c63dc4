"""Sizes whose products pass 32 bits are refused by the paged cache's calls and by their
host arithmetic, before anything is launched (CPU: the pointers given would fault)."""

import ctypes

import pytest

from paper_2608_26140_amd import acache as A
from tests.test_paged_host import append, attention, cache


def host(d, c, per):
    """(workspace bytes, status and splits of the schedule)."""
    n = ctypes.c_int32(-1)
    d, c = ctypes.byref(d), ctypes.byref(c)
    size = A.lib.acache_paged_workspace_size(d, c, per, 0)
    return size, A.lib.acache_paged_attention_schedule(d, c, per, 0, 1 << 60, ctypes.byref(n)), n.value


@pytest.mark.parametrize("per", [16384, 1 << 20, 1 << 22, 3 << 21, 1 << 23, (1 << 24) - 1])
def test_more_tiles_than_a_launch_has(per):
    """512 queries of the one KV head in each row: 2^21 tiles of four and more, with 2^31 and 2^32 queries among them."""
    d = A.make_dims(1024, 512, 1, 2, 256, "f32")
    c = cache(batch=1, ld=2)
    assert attention(c=c, d=d, per=per) == 4
    assert host(d, c, per) == (0, 4, 0)


def test_the_most_tiles_that_are_taken():
    d = A.make_dims(1024, 512, 1, 2, 256, "f32")
    size, status, splits = host(d, cache(batch=1, ld=2), 16383)
    assert size >= 256 and status == 0 and splits >= 1


@pytest.mark.parametrize("per", [1, 5])
def test_rows_of_heads_past_32_bits(per):
    for d, c in ((A.make_dims(256, 1 << 24, 1, 128, 256, "bf16"), cache(batch=1, ld=128)),
                 (A.make_dims(256, 1 << 30, 1, 2, 256, "f32"), cache(batch=1, ld=2))):
        assert append(c=c, d=d, per=per, q_ld=1 << 31, q_out_ld=1 << 31) == 4
        assert attention(c=c, d=d, per=per, q_ld=1 << 31, out_ld=1 << 31) == 4
        assert host(d, c, per)[:2] == (0, 4)
