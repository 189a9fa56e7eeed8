"""The choice of beams where scores are equal in fp64 and logits are not: the larger
logit of a beam comes first, the lower beam before the others."""

import math

import pytest
import torch

from tests.paged_util import DEV
from tests.test_gpu_beam import Beam, logits

pytestmark = pytest.mark.gpu


def best_of(row, n):
    """Tokens of a row by value, equal ones by place."""
    x = row.float().cpu().tolist()
    return sorted((v for v in range(len(x)) if x[v] > -math.inf), key=lambda v: (-x[v], v))[:n]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("w", [1, 2, 4, 16])
def test_scores_that_outweigh_the_logits(dtype, w):
    """All scores of a request are 1e30 below zero: equal whatever the logits add."""
    for v in (1, 3, 100, 5003, 40000) + (600000,) * (w <= 2):
        x, _ = logits(2, w, v, dtype, 10 * w)
        x[0, 0, ::2] = -math.inf
        y = Beam(x, torch.full((2, w), -1e30, device=DEV)).run().check()
        for b in range(2):
            want = [(i, t) for i in range(w) for t in best_of(x[b, i], w)][:w]
            want += [(-1 - b * w, -1)] * (w - len(want))
            assert list(zip(y.parent[b].tolist(), y.token[b].tolist())) == [(b * w + i, t)
                                                                            for i, t in want]


@pytest.mark.parametrize("v", [10, 3000, 40000, 600000])
def test_logits_whose_differences_are_below_a_scores_step(v):
    """Logits of 1e-20 and 2e-20 beside zeros."""
    x = torch.zeros((1, 2, v), device=DEV)
    x[0, 0, 5], x[0, 0, v - 1] = 1e-20, 2e-20
    y = Beam(x, torch.tensor([[0.0, -1.0]], device=DEV)).run().check()
    assert y.token.tolist() == [[v - 1, 5]] and y.parent.tolist() == [[0, 0]]
    y = Beam(x[:, :1], torch.zeros((1, 1), device=DEV)).run().check()
    assert y.token.tolist() == [[v - 1]]


def test_the_lower_beam_comes_first_whatever_its_logits():
    """Rows that differ by a shift: equal scores, other logits."""
    g = torch.Generator().manual_seed(4)
    x = (torch.randint(-40, 41, (1, 1, 700), generator=g) / 4).repeat(1, 3, 1).to(DEV)
    x[0, 0, 1:] -= 1000  # one value stands out, so its row's sum is 1
    x[0, 1], x[0, 2] = x[0, 0] + 64, x[0, 0] - 64
    y = Beam(x, torch.zeros((1, 3), device=DEV)).run().check()
    assert y.parent.tolist() == [[0, 1, 2]] and y.token.tolist() == [[0, 0, 0]]
