"""The confidence of a drawn token is its softmax probability at temperature 1: tokens
that weigh nothing at the temperature drawn with count there."""

import math

import pytest
import torch

from tests.test_gpu_sample import BF, F32, check

pytestmark = pytest.mark.gpu


def rows_of(n, dt):
    """The largest logit between -511 and -453, the others -512 and below, ordinary ones, masked ones."""
    x = torch.empty(7, n)
    for r, m in enumerate((-500.0, -505.0, -493.0, -511.0, -453.0)):
        x[r] = -512.0
        x[r, (7 * r + 3) % n] = m
    x[5] = -512.0 - 4.0 * (torch.arange(n) % 5)
    x[5, n // 2] = -508.0
    x[6] = -530.0
    x[6, ::3] = -math.inf
    x[6, 1 % n] = -509.0
    x[6, n - 1] = math.nan
    return x.to(dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("n", [5, 2003, 126464])
def test_distant_logits_count_at_temperature_1(dt, n):
    x = rows_of(n, dt)
    rows = x.shape[0]
    for t in (0.01, 0.02, 0.1, 0.3, 1.0, 1.7):
        check(x, [0.2] * rows, t=[t] * rows, what=f"temperature {t}")
        check(x, [0.9] * rows, t=[t] * rows, k=[3] * rows, p=[0.8] * rows, m=[0.01] * rows, what=f"temperature {t}, cuts")
    check(x, [0.5] * rows, t=[0.0] * rows, what="greedy")
