"""The reference of the choice of beams where logits are large, against rational
arithmetic on the arguments of its exponentials."""

import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import paged


@pytest.mark.parametrize("size", [1.0, 1e9, 4e13, 4e16, 4e18, 1e33, 3e38])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_keep_what_large_logits_would_round_away(size, sign):
    """Every row has its maximum several times: a score is the beam's and minus the log
    of their number."""
    rng = np.random.default_rng(3)
    w, v = 4, 50
    top = np.float32(sign * size)
    step = np.abs(np.spacing(top)) * 2.0 ** 10  # below the top by this or more
    x = top.astype(np.float64) - step * rng.integers(1, 50, (w, v))
    for i in range(w):
        x[i, rng.permutation(v)[:i + 1]] = top
    s = -20 * rng.random(w)
    every = []
    for i in range(w):
        high = max(Fraction(y) for y in x[i])
        total = math.fsum(math.exp(max(-1e4, float(Fraction(y) - high))) for y in x[i])
        every += [(s[i] - math.log(total) + float(Fraction(y) - high), i, j)
                  for j, y in enumerate(x[i])]
    want = sorted(every, key=lambda c: (-c[0], c[1], c[2]))[:w]
    got = paged.beam(x, s)
    for (z, i, j), (gz, gi, gj) in zip(want, got):
        assert (gi, gj) == (i, j) and abs(gz - z) <= 1e-13 * (1 + abs(z))
