"""Drawn tokens on a stream of their own: the settings are there when another stream reads
them and stay until it has, and every commit has numbers of its own."""

import pytest
import torch

import workloads as W
from paper_2608_26140_amd import acache as A
from paper_2608_26140_amd import driver as D
from paper_2608_26140_amd import workload as WL
from tests.test_gpu_result_streams import stream_of

pytestmark = pytest.mark.gpu

BLOCK, VOCAB = 8, 1024
SETTINGS = dict(temperature=[0.6, 1.0, 0.0], top_k=[40, 0, 3], top_p=[0.9, 1.0, 0.5], min_p=[0.0, 0.01, 0.0])


def setup():
    batch = WL.build(W.get_config("mini-serve"), keep_host=False).batch
    assert batch.B == 3
    logits = 3 * torch.randn(batch.B * BLOCK, VOCAB, generator=seeded(3), device="cuda")
    want = D.Sampling(batch, BLOCK, **SETTINGS, generator=seeded(5)).commit(logits)
    torch.cuda.synchronize()
    return batch, logits, want


def seeded(n):
    return torch.Generator(device="cuda").manual_seed(n)


def scrap(batch):
    """What the settings' memory held and holds otherwise: as much, in as many tensors, of another value."""
    return [torch.full((batch.B * BLOCK,), 7.0, device="cuda") for _ in range(64)]


def test_settings_are_there_when_another_stream_reads_them():
    batch, logits, want = setup()
    side, generator = torch.cuda.Stream(), seeded(5)
    given = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda") for n, v in SETTINGS.items()}
    before = scrap(batch)
    torch.cuda.synchronize()
    del before
    torch.cuda._sleep(20_000_000)
    sampling = D.Sampling(batch, BLOCK, **given, generator=generator)
    got = sampling.commit(logits, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_settings_stay_until_another_stream_has_read_them():
    batch, logits, want = setup()
    side, generator = torch.cuda.Stream(), seeded(5)
    sampling = D.Sampling(batch, BLOCK, **SETTINGS, generator=generator)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = sampling.commit(logits, stream=side)
    del sampling
    after = scrap(batch)
    torch.cuda.current_stream().synchronize()
    side.synchronize()
    assert torch.equal(got, want) and all((t == 7).all() for t in after)


def test_numbers_are_a_commits_own(monkeypatch):
    """Two commits of one object, on two streams at once: neither draws with the other's numbers."""
    batch, logits, want = setup()
    taken = []
    call = A.acache_sample_commit
    monkeypatch.setattr(A, "acache_sample_commit", lambda x, u, *a, **k: (taken.append(u), call(x, u, *a, **k))[1])
    side, generator = torch.cuda.Stream(), seeded(5)
    sampling = D.Sampling(batch, BLOCK, **SETTINGS, generator=generator)
    got = sampling.commit(logits), sampling.commit(logits, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want)
    here, there = taken
    assert here.data_ptr() != there.data_ptr() and not torch.equal(here, there)
    assert stream_of(here) == torch.cuda.current_stream().cuda_stream and stream_of(there) == side.cuda_stream
    again = call(logits, there, **sampling.settings)
    assert torch.equal(got[1], again)


def test_captured_commits_draw_anew():
    """Replays of a captured commit draw what eager ones draw from the same seeds."""
    batch, logits, _ = setup()
    sampling = D.Sampling(batch, BLOCK, **SETTINGS)
    out = torch.empty(batch.B * BLOCK, dtype=torch.int32, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sampling.commit(logits, out=out)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        sampling.commit(logits, out=out)
    for seed in (1, 2, 1, 3):
        torch.cuda.manual_seed(seed)
        want = sampling.commit(logits)
        out.zero_()
        torch.cuda.manual_seed(seed)
        graph.replay()
        assert torch.equal(out, want)
        torch.cuda.synchronize()
