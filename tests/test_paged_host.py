"""What the paged cache's calls and the sampled commit refuse, before anything is launched
(CPU: the pointers given would fault), and their host arithmetic."""

import ctypes

import pytest
import torch

from paper_2608_26140_amd import acache as A

BF = torch.bfloat16
P = ctypes.c_void_p(256)


def dims(dt="bf16", H=8, G=2, d=128):
    return A.make_dims(H * d, H, G, d, 256, dt)


def cache(batch=2, max_blocks=4, block=16, n_blocks=10, ld=256, table_ld=4, k=256, v=256, tables=256):
    return A.PagedCacheDesc(k, v, ld, n_blocks, tables, table_ld, batch, max_blocks, block)


def append(c=None, d=None, per=3, q=P, q_ld=1024, k=P, k_ld=256, v=P, v_ld=256, pos=P, q_out=P, q_out_ld=1024):
    return A.lib.acache_paged_append(ctypes.byref(d or dims()), ctypes.byref(c or cache()), per, q, q_ld, k, k_ld, v, v_ld,
                                     pos, None, q_out, q_out_ld, None)


def attention(c=None, d=None, per=3, q=P, q_ld=1024, key_len=P, out=P, out_ld=1024, ws=None, ws_bytes=0):
    return A.lib.acache_paged_attention(ctypes.byref(d or dims()), ctypes.byref(c or cache()), per, q, q_ld, key_len, 0, out,
                                        out_ld, None, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [append, attention])
def test_cache_checks(call):
    assert call(c=cache(batch=-1)) == 2 and call(per=-1) == 2
    assert call(c=cache(block=0)) == 2
    assert call(c=cache(n_blocks=0)) == 2
    assert call(c=cache(table_ld=3)) == 2                      # shorter than a table
    assert call(c=cache(ld=248)) == 2                          # shorter than a row
    assert call(c=cache(n_blocks=1 << 27)) == 4                # 2^31 slots
    assert call(c=cache(max_blocks=1 << 27, table_ld=1 << 27)) == 4
    assert call(c=cache(batch=1 << 20), per=1 << 10) == 4
    assert call(c=cache(batch=1 << 20), per=16) == 4           # 2^24 rows
    assert call(c=cache(k=None)) == 1 and call(c=cache(v=None)) == 1 and call(c=cache(tables=None)) == 1
    assert call(c=cache(k=264)) == 3 and call(c=cache(ld=260)) == 3
    assert call(d=dims(d=64)) == 4                             # bf16 heads are of 128
    assert call(c=cache(batch=0)) == 0 and call(per=0) == 0    # nothing to do


def test_append_checks():
    assert append(k=None) == 1 and append(v=None) == 1 and append(pos=None) == 1
    assert append(q_out=None) == 1
    assert append(k_ld=128) == 2 and append(v_ld=128) == 2 and append(q_ld=1016) == 2 and append(q_out_ld=1016) == 2
    assert append(q_ld=1032) == 2                              # q_out is q, with another stride
    assert append(q=ctypes.c_void_p(264)) == 3 and append(k_ld=260) == 3 and append(q_out_ld=1028) == 3


def test_attention_checks():
    assert attention(q=None) == 1 and attention(out=None) == 1 and attention(key_len=None) == 1
    assert attention(q_ld=1016) == 2 and attention(out_ld=1000) == 2
    assert attention(c=cache(batch=1 << 20), d=dims("f32"), per=8) == 4  # 2^24 tiles of four queries
    assert attention(out=ctypes.c_void_p(260)) == 3 and attention(ws=ctypes.c_void_p(260), ws_bytes=1 << 20) == 3


def test_sample_checks():
    def call(dtype=1, x=P, ld=100, rows=3, n=100, u=P, out=P, pos=None, ids=None, ids_len=0):
        return A.lib.acache_sample_commit(dtype, x, ld, rows, n, None, None, None, None, u, out, None, None, pos, ids,
                                          ids_len, None)
    assert call(dtype=7) == 4
    assert call(rows=-1) == 2 and call(n=-1) == 2 and call(ld=99) == 2 and call(ids_len=-1) == 2 and call(n=0, ld=0) == 2
    assert call(n=(1 << 19) + 1, ld=1 << 20) == 4 and call(rows=1 << 22) == 4
    assert call(x=None) == 1 and call(u=None) == 1 and call(out=None) == 1 and call(pos=P) == 1
    assert call(rows=0) == 0


def test_workspace_and_splits():
    """A call splits its keys with the workspace it asks for, in fewer parts with less, and not without."""
    for batch, per, H, G in ((1, 1, 32, 32), (8, 1, 28, 4), (1, 1, 8, 1), (4, 32, 28, 4)):
        d = dims(H=H, G=G)
        c = cache(batch=batch, max_blocks=400, block=64, n_blocks=batch * 400, ld=G * 128, table_ld=400)
        size = A.lib.acache_paged_workspace_size(ctypes.byref(d), ctypes.byref(c), per, 0)

        def splits(n, max_len=0):
            out = ctypes.c_int32(-1)
            assert A.lib.acache_paged_attention_schedule(ctypes.byref(d), ctypes.byref(c), per, max_len, n, ctypes.byref(out)) == 0
            return out.value
        full = splits(size)
        assert full >= 1 and splits(0) == 1 and splits(1 << 60) == full
        assert splits(size, max_len=100) == 1
        each = batch * per * H * 130 * 4
        assert size >= (full * each if full > 1 else 0)
        for n in range(1, full):
            assert 1 <= splits(n * each) <= n and splits(n * each + each - 1) == splits(n * each)
    c = cache(batch=0)
    assert A.lib.acache_paged_workspace_size(ctypes.byref(dims()), ctypes.byref(c), 3, 0) == 256
    c = cache(block=0)
    assert A.lib.acache_paged_workspace_size(ctypes.byref(dims()), ctypes.byref(c), 3, 0) == 0


def test_binding_refusals():
    """The binding refuses what it can see: types, shapes, strides, devices."""
    k, v = torch.zeros(64, 256, dtype=BF), torch.zeros(64, 256, dtype=BF)
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(TypeError):
        A.PagedCache(k.half(), v.half(), 16, t)
    with pytest.raises(TypeError):
        A.PagedCache(k.t(), v.t(), 16, t)
    with pytest.raises(TypeError):
        A.PagedCache(k, v, 16, t.long())
    with pytest.raises(TypeError):
        A.PagedCache(k, v, 16, t.t())
    with pytest.raises(ValueError):
        A.PagedCache(k, v[:32], 16, t)
    with pytest.raises(ValueError):
        A.PagedCache(k, v.float(), 16, t)
    for block in (0, -1, 65):
        with pytest.raises(ValueError):
            A.PagedCache(k, v, block, t)
    c, d = A.PagedCache(k, v, 16, t), dims()
    rows, i = torch.zeros(6, 256, dtype=BF), torch.zeros(6, dtype=torch.int32)
    q = torch.zeros(6, 1024, dtype=BF)
    with pytest.raises(TypeError):
        A.acache_paged_append(d, c, rows[:5], rows, i, 3)
    with pytest.raises(TypeError):
        A.acache_paged_append(d, c, rows.float(), rows, i, 3)
    with pytest.raises(TypeError):
        A.acache_paged_append(d, c, rows, rows, i.long(), 3)
    with pytest.raises(TypeError):
        A.acache_paged_append(d, c, rows, rows, i, 3, at=i[:4])
    with pytest.raises(ValueError):
        A.acache_paged_append(d, c, rows, rows, i, 3, q_out=q)
    with pytest.raises(ValueError):  # not on a GPU
        A.acache_paged_append(d, c, rows, rows, i, 3)
    with pytest.raises(ValueError):  # more heads than the pools' rows hold
        A.acache_paged_append(dims(H=16, G=4), c, torch.zeros(6, 512, dtype=BF), torch.zeros(6, 512, dtype=BF), i, 3)
    with pytest.raises(TypeError):
        A.acache_paged_attention(d, c, q[:, :1016], i, 3)
    with pytest.raises(TypeError):
        A.acache_paged_attention(d, c, q, i, 3, out=q.float())
    with pytest.raises(TypeError):
        A.acache_paged_attention(d, c, q, i, 3, out=q, lse=torch.zeros(6))
    x, u = torch.zeros(3, 10, dtype=BF), torch.zeros(3, dtype=torch.float64)
    with pytest.raises(TypeError):
        A.acache_sample_commit(x.half(), u)
    with pytest.raises(TypeError):
        A.acache_sample_commit(x, u.float())
    with pytest.raises(TypeError):
        A.acache_sample_commit(x, u, temperature=torch.ones(2))
    with pytest.raises(TypeError):
        A.acache_sample_commit(x, u, top_k=torch.ones(3))
    with pytest.raises(ValueError):
        A.acache_sample_commit(x, u, commit_pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):  # not on a GPU
        A.acache_sample_commit(x, u)


def test_struct_layout():
    """PagedCacheDesc has the C struct's layout."""
    import os
    import shutil
    import subprocess
    import tempfile
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f for f, _ in A.PagedCacheDesc._fields_]
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "l.c"), os.path.join(tmp, "l")
        open(src, "w").write('#include <stddef.h>\n#include <stdio.h>\n#include "acache.h"\nint main(void) {\n' + "".join(
            f'printf("%zu\\n", offsetof(acache_paged_cache, {n}));' for n in names) +
            'printf("%zu\\n", sizeof(acache_paged_cache)); return 0; }\n')
        subprocess.run(["gcc", "-std=c11", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I",
                        "/opt/rocm/include", src, "-o", exe], check=True)
        got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [getattr(A.PagedCacheDesc, n).offset for n in names] + [ctypes.sizeof(A.PagedCacheDesc)]
