"""The tree oracle itself: by hand, against torch, and by its own statistics."""

import math
import random

import numpy as np
import torch

from oracle import fp8 as ofp8
from oracle import tree as otree


def test_lines():
    parents = [-1, 0, 0, 1, 3, 2]
    assert [otree.line(parents, i) for i in range(6)] == [
        [0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0, 2, 5]]
    assert otree.chain(3) == [-1, 0, 1]


def test_keys_by_hand():
    parents = [-1, 0, 0, 1]
    assert otree.keys_of(parents, 3, 5, 2, 0, None) == ([-2, -1, 0, 1, 2, 3, 4], [0, 1, 3])
    # window of 3 with one sink, position 7: prompt, sink 0, positions 5, 6, 7
    assert otree.keys_of(parents, 3, 5, 2, 1, 3) == ([-2, -1, 0], [0, 1, 3])
    assert otree.keys_of(parents, 1, 5, 2, 1, 3) == ([-2, -1, 0, 4], [0, 1])
    # a chunk that starts inside the prompt: its prompt tokens stay in reach
    assert otree.keys_of(otree.chain(5), 4, -1, 2, 0, 2) == ([-2], [0, 3, 4])


def test_attend_is_softmax_attention():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(n, 16, generator=g, dtype=torch.float64) for n in (1, 33, 33))
    out, band = otree.attend(q[0].numpy(), k.numpy(), v.numpy(), 0.25)
    ref = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None], scale=0.25)
    assert np.abs(out - ref[0, 0].numpy()).max() < 1e-14
    # fp32 arithmetic stays inside the bound
    s = (k.float() @ q[0].float()) * 0.25
    w = torch.exp(s - s.max())
    o = (w @ v.float()) / w.sum()
    assert np.abs(o.double().numpy() - out).max() <= band * v.abs().max().item()


def test_verify_by_hand():
    t = np.array([[0.5, 0.25, 0.25], [0.0, 1.0, 0.0], [0.1, 0.2, 0.7]], dtype=np.float32)
    d = np.array([[0.25, 0.5, 0.25]] * 3, dtype=np.float32)
    parents = [-1, 0, 0]
    # token 1: 0.25 / 0.5; accepted below 0.5
    assert otree.verify(parents, [0, 1, 0], t, d, [0, 0.49, 0, 0.5], 3) == ([0, 1], 1)
    # rejected: the residual is all on token 0, and the second child is token 0
    assert otree.verify(parents, [0, 1, 0], t, d, [0, 0.5, 0.99, 0.05], 3) == ([0, 2], 0)
    # both rejected (token 2 is not in the residual): token 0 follows
    assert otree.verify(parents, [0, 1, 2], t, d, [0, 0.5, 0.0, 0.99], 3) == ([0], 0)
    # certain drafts: token 1 with 1/4, then token 2 with 1/3 of what is left
    assert otree.verify(parents, [0, 1, 2], t, None, [0, 0.25, 0.33, 0.8], 3) == ([0, 2], 2)
    assert otree.verify(parents, [0, 1, 2], t, None, [0, 0.25, 0.34, 0.8], 3) == ([0], 0)
    assert otree.verify(parents, [0, 1, 2], t, None, [0, 0, 0, 0], 0) == ([], -1)


def test_verify_keeps_the_targets_distribution():
    rng = random.Random(1)
    t = np.array([[0.4, 0.1, 0.3, 0.2]] * 3, dtype=np.float32)
    d = np.array([[0.1, 0.4, 0.1, 0.4]] * 3, dtype=np.float32)
    n, seen = 20000, np.zeros(4)
    for _ in range(n):
        x = rng.choices(range(4), d[0], k=3)
        path, nxt = otree.verify([-1, 0, 0], x, t, d, [rng.random() for _ in range(4)], 3)
        seen[x[path[1]] if len(path) > 1 else nxt] += 1
    p = t[0].astype(np.float64)
    assert (np.abs(seen / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


def test_encode_inverts_decode_and_rounds_to_nearest_even():
    codes = np.array([c for c in range(256) if c & 0x7F != 0x7F], dtype=np.uint8)
    assert (otree.encode_e4m3(ofp8.decode_e4m3(codes)) == codes).all()
    x = torch.randn(50000, generator=torch.Generator().manual_seed(0)) * 30
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (otree.encode_e4m3(x.numpy()) == want).all()
    assert otree.encode_e4m3(math.nan) == 0x7F and otree.encode_e4m3(1e30) == 0x7E
