"""Results that a call on another stream makes for itself are that stream's
memory: freed, they are its to take again, and not the current stream's."""

import pytest
import torch

from paper_2608_26140_amd import acache as A
from tests.gpu_util import up_i32

pytestmark = pytest.mark.gpu

BF, N, D = torch.bfloat16, 600, 4096


def rows(n=N, d=D):
    return torch.randn(n, d, device="cuda").to(BF)


def calls():
    dims = A.make_dims(D, 32, 32, 128, 256, "bf16")
    at = up_i32(range(N))
    x, w, k, v = rows(), rows(512), rows(), rows()
    scores = torch.rand(1000, 1000, device="cuda")
    lay = A.Layout(3000, 0, 1000, 2900, 100, 0, 1000, 3000)
    paged = dict(block_size=100, shared_blocks=up_i32(range(10)), private_blocks=up_i32(range(10, 10 + 64 * 20)),
                 blocks_per_request=20)
    fresh = at.view(1, N)
    return {
        "topk": lambda s: A.acache_topk(scores, 600, stream=s),
        "gather_rows": lambda s: A.acache_gather_rows(x, at, stream=s),
        "build_maps": lambda s: A.acache_build_maps(lay, 64, None, 0, stream=s)["read_slots"],
        "build_maps_paged": lambda s: A.acache_build_maps_paged(lay, 64, None, 0, **paged, stream=s)["read_slots"],
        "attention": lambda s: A.acache_attention(dims, [0, N], [0, N], x, at, k, v, stream=s),
        "rmsnorm": lambda s: A.acache_rmsnorm(dims, x, w[0], stream=s),
        "linear": lambda s: A.acache_linear(dims, x, w, stream=s),
        "kv_deviation": lambda s: A.acache_kv_deviation(dims, k, v, fresh, at, stream=s),
        "argmax_commit": lambda s: A.acache_argmax_commit(x, stream=s),
    }


def stream_of(t):
    """The stream whose memory pool t lies in."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not in any segment")


def test_results_belong_to_the_stream_of_the_call():
    side = torch.cuda.Stream()
    here = torch.cuda.current_stream().cuda_stream
    assert side.cuda_stream != here
    for name, call in calls().items():
        print(name, flush=True)
        want = call(None)
        torch.cuda.synchronize()
        got = call(side)
        side.synchronize()
        assert torch.equal(got, want), name
        assert stream_of(want) == here and stream_of(got) == side.cuda_stream, name
