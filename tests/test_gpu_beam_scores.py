"""The choice of beams where logits are large: scores are not rounded away against
them."""

import pytest
import torch

from tests.paged_util import DEV
from tests.test_gpu_beam import Beam, logits

pytestmark = pytest.mark.gpu

SIZES = [1e3, 1e9, 4e13, 4e16, 4e18, 1e33, 3e38]


def rows_with_equal_tops(b, w, v, size, seed):
    """fp32 logits; row ``i`` of a request has its maximum ``i + 1`` times, other values a
    thousand units in the last place below it or more, all over the row."""
    g = torch.Generator().manual_seed(seed)
    top = torch.tensor(size, dtype=torch.float32)
    step = (torch.nextafter(top, top * 2) - top).abs().double() * 2 ** 10
    x = top.double() - step * torch.randint(1, 1000, (b, w, v), generator=g)
    for r in range(b):
        for i in range(w):
            x[r, i, torch.randperm(v, generator=g)[:i + 1]] = top.double()
    return x.float().to(DEV), (-20 * torch.rand((b, w), generator=g)).to(DEV)


@pytest.mark.parametrize("size", SIZES + [-s for s in SIZES])
def test_rows_of_large_logits(size):
    for b, w, v in ((2, 4, 4000), (1, 1, 17), (3, 8, 20000)):
        Beam(*rows_with_equal_tops(b, w, v, size, w)).run().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("spread", [1e4, 1e9, 1e18, 1e33])
def test_logits_far_apart(dtype, spread):
    """The best of every beam is its whole distribution: the beams' own scores."""
    x, s = logits(2, 4, 4000, torch.float32, 6)
    y = Beam((x * spread).to(dtype), s).run().check()
    if spread > 1e8:
        assert torch.equal(y.next, s.sort(1, descending=True).values)


def test_a_shift_of_all_logits_changes_nothing():
    """Logits that a shift of 2^20 does not round (quarters) have the same scores."""
    g = torch.Generator().manual_seed(2)
    x = (torch.randint(-40, 41, (2, 4, 9000), generator=g) / 4).to(DEV)
    s = (-20 * torch.rand((2, 4), generator=g)).to(DEV)
    want = Beam(x, s).run().check()
    for shift in (2.0 ** 20, -2.0 ** 20):
        y = Beam(x + shift, s).run().check()
        assert all(torch.equal(p, q) for p, q in ((y.next, want.next), (y.parent, want.parent),
                                                  (y.token, want.token)))


def test_rows_at_different_heights():
    """Rows that differ by a shift alone tie: the first beam's places come first."""
    g = torch.Generator().manual_seed(4)
    x = (torch.randint(-40, 41, (1, 1, 3000), generator=g) / 4).repeat(1, 4, 1).to(DEV)
    x += torch.tensor([0.0, 1e6, -1e6, 2e6], device=DEV)[None, :, None]
    assert (x[0, 0] == x[0, 0].max()).sum() >= 4
    y = Beam(x, torch.zeros((1, 4), device=DEV)).run().check()
    assert y.parent.tolist() == [[0, 0, 0, 0]]
