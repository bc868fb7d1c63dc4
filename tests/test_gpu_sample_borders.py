"""Sampled commits whose cuts end at a token that shares its bin with none."""

import pytest
import torch

from tests.test_gpu_sample import BF, F32, check, uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("n", [40, 5003, 50021])
def test_borders_of_one_token(dt, n):
    """The 30 largest logits, in any order, a quarter apart: every top-k border of up to 30 tokens and every top-p border
    is one of them, and so is the token drawn."""
    rows = 60
    g = torch.Generator().manual_seed(n)
    x = -6 - torch.rand(rows, n, generator=g)
    for r in range(rows):
        x[r, torch.randperm(n, generator=g)[:30]] = 8 - 0.25 * torch.arange(30)
    x, u = x.to(dt), uniform(rows, n + 1)
    k, p = [1 + r % 30 for r in range(rows)], [(r + 0.4) / (rows + 20) for r in range(rows)]
    check(x, u, k=k, what="top-k")
    check(x, u, p=p, what="top-p")
    check(x, u, t=[0.5 + r / 40 for r in range(rows)], k=k, p=p, m=[0.003] * rows, what="all")
