"""Slots that a tree call leaves alone or shares: rows of a ring, unused requests."""

import random

import pytest
import torch

from tests.test_gpu_tree_verify_append import Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,layers", [("bf16", None), ("fp8", 2)])
@pytest.mark.parametrize("ring,sinks", [(12, 4), (15, 0)])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_ring_slots_take_the_last_row_that_is_written(seed, ring, sinks, kv, layers):
    """More accepted rows than ring slots, some of their path entries outside the
    nodes: a skipped entry leaves its slot to the last one before it."""
    rng = random.Random(seed)
    a = Append(mode="window", n_att=12, sinks=sinks, ring=ring, nodes=40, bases=[0, 1, -13], kv=kv,
               layers=layers, seed=seed)
    a.path = [[rng.choice([rng.randrange(40), rng.choice([-1, 40, 1 << 30, -(1 << 31)])])
               for _ in range(40)] for _ in range(3)]
    a.path[1][20:] = [-1] * 20  # nothing valid in the slots' last rows, nor before
    a.path[2] = list(range(30)) + [-1] * 10
    a.accepted = [40, 40, 40]
    a.check()
    a.counts = [40, 25, 33]  # entries past a request's count are skipped as well
    a.check()


def test_ring_slots_of_a_wholly_skipped_slot_stay():
    a = Append(mode="window", n_att=12, sinks=4, ring=12, nodes=40, bases=[0, 1, -13])
    a.path = [[-1] * 40, [0] + [99] * 39, [-7] * 39 + [3]]
    a.accepted = [40, 40, 40]
    a.check()
