"""Slots that a tree call leaves alone or shares: rows of a ring, unused requests."""

import random

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.gpu_util import DEV
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


def test_unused_slots_stay_unused_over_steps():
    """A slot of count 0, its base below the prompt: nothing of it is accepted, so
    its base stays where it is and its caches as they are, step after step; a
    slot marked by its base alone is one to the attention and the append."""
    batch, n, vocab, prompt = 3, 4, 17, 9
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    p = B.make_params(prompt, 6, 6, 1, 1, B.MODE_DENSE)
    s = B.make_shape(batch, 2, 2, 64)
    g = torch.Generator().manual_seed(2)
    rand = lambda *shape: torch.randn(shape, generator=g).bfloat16().to(DEV)  # noqa: E731
    k, v = rand(batch, 2, prompt + 36, 64), rand(batch, 2, prompt + 36, 64)
    lay, k0, v0 = B.kv_layout(k), k.clone(), v.clone()
    base, count, parent = ints([0, -prompt - 1, 3]), ints([n, 0, n]), ints([[-1, 0, 0, 1]] * batch)
    plan = torch.empty(B.tree_plan_bytes(batch, n), dtype=torch.uint8, device=DEV)
    size = B.tree_workspace_bytes(p, s, n)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None
    path = torch.empty((batch, n), dtype=torch.int32, device=DEV)
    got, tok = (torch.empty(batch, dtype=torch.int32, device=DEV) for _ in range(2))
    for step in range(4):
        x = rand(batch, n, 6, 64)
        out = torch.full((batch, n, 2, 64), 7.0, device=DEV)
        B.tree_plan(parent, count, plan)
        tree = B.make_tree(n, base, count, plan)
        B.tree_attention(p, s, tree, x[:, :, :2], x[:, :, 2:4], x[:, :, 4:], k, v, lay, 0.125, out,
                         ws)
        target = torch.softmax(torch.randn((batch, n, vocab), generator=g), -1).to(DEV)
        B.tree_verify(tree, ints([[1, 2, 3, 4]] * batch), target, None,
                      torch.rand((batch, n + 1), generator=g).to(DEV), path, got, tok)
        B.kv_append(p, s, tree, x[:, :, 2:4], x[:, :, 4:], k, v, lay, path, got)
        base += got
        assert (out[1] == 7.0).all() and int(got[1]) == 0 and int(tok[1]) == -1
        assert (path[1] == -1).all() and int(base[1]) == -prompt - 1
        assert (got[[0, 2]] >= 1).all() and (tok[[0, 2]] >= 0).all()
    assert torch.equal(k[1], k0[1]) and torch.equal(v[1], v0[1])
    assert not torch.equal(k[0], k0[0]) and not torch.equal(k[2], k0[2])
    # by its base alone
    k0, out = k.clone(), torch.full((batch, n, 2, 64), 7.0, device=DEV)
    tree = B.make_tree(n, base, None, plan)
    B.tree_attention(p, s, tree, x[:, :, :2], x[:, :, 2:4], x[:, :, 4:], k, v, lay, 0.125, out, ws)
    B.kv_append(p, s, tree, x[:, :, 2:4], x[:, :, 4:], k, v, lay)
    assert (out[1] == 7.0).all() and (out[[0, 2]] != 7.0).any() and torch.equal(k[1], k0[1])
