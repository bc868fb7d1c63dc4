"""Drawn tokens on a stream of their own."""

import pytest
import torch

import workloads as W
from paper_2608_26140_amd import driver as D
from paper_2608_26140_amd import workload as WL

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
