"""Pins of the references for paged caches and beams."""

import math
import random

import numpy as np

from oracle import paged


def test_update_worked_example():
    table, refs = [[3, 1, -1], [3, -1, -1], [-1, -1, -1]], [0, 1, 0, 2, 0]
    cursor, slots, pos, copies, flags = paged.update(table, refs, 4, [2, 2, 2], [3, 3, -1], [2, 1, 0],
                                                     2, 4)
    # request 0 writes rows 3 and 4: page 3 is shared, page 1 its own; request 1 row 3
    assert table == [[4, 1, -1], [0, -1, -1], [-1, -1, -1]]
    assert refs == [1, 1, 0, 0, 1] and cursor == 1
    assert slots == [[19, 4], [3, -1], [-1, -1]]
    assert pos == [2, 1, -1] and copies == [[3, 4, 3], [3, 0, 3], [-1, -1, -1]]
    assert flags == [0, 0, 0]


def test_window_positions_are_all_that_is_left():
    """Every row that a later step attends keeps its page; the others' whole pages go."""
    rng = random.Random(2)
    for _ in range(200):
        page, prompt, sinks = rng.choice([1, 2, 4, 8]), rng.randrange(0, 12), rng.randrange(0, 5)
        n_att = sinks + rng.randrange(1, 12)
        width = 60 // page + 1
        table, refs, cursor = [[-1] * width], [0] * width, 0
        length = 0
        while length < 50:
            new = rng.randrange(1, 5)
            cursor, _, _, _, flags = paged.update(table, refs, cursor, [prompt], [length], [new], 4,
                                                  page, sinks, n_att - sinks)
            assert flags == [0]
            first = length - prompt  # positions of the new rows
            length += new
            need = set(range(min(prompt, length)))
            for t in range(max(first, 0), length - prompt):
                need |= {prompt + j for j in paged.attended_positions("window", t, n_att, sinks)}
            held = {i for i, g in enumerate(table[0]) if g >= 0}
            assert {r // page for r in need} <= held
            lo, hi = prompt + sinks, length - new - (n_att - sinks) + 1
            assert held == {i for i in range(-(-length // page))
                            if not (i * page >= lo and (i + 1) * page <= hi)}
            assert sum(refs) == len(held)


def test_reorder_counts():
    table, refs = [[0, 1], [2, -1], [0, 3]], [2, 1, 1, 1]
    assert paged.reorder(table, refs, [2, 2, -1]) == [[0, 3], [0, 3], [-1, -1]]
    assert refs == [2, 0, 0, 2]


def test_attention_is_the_decode_reference():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal(64), rng.standard_normal((40, 64)), rng.standard_normal((40, 64))
    out, z, mass = paged.attention(q, k, v, 0.125)
    w = np.exp(0.125 * (k @ q))
    np.testing.assert_allclose(out, (w / w.sum()) @ v, rtol=1e-12)
    assert (mass >= np.abs(out) - 1e-15).all() and np.allclose(z, 0.125 * (k @ q))
    assert (paged.attention(q, k[:0], v[:0], 1.0)[0] == 0).all()


def test_beam_against_enumeration():
    rng = np.random.default_rng(1)
    for _ in range(50):
        w, v = int(rng.integers(1, 5)), int(rng.integers(1, 9))
        x, s = rng.integers(-2, 3, (w, v)).astype(float), rng.integers(-2, 1, w).astype(float)
        x[rng.random((w, v)) < 0.2] = -math.inf
        every = []
        for i in range(w):
            total = sum(math.exp(y) for y in x[i])
            for j in range(v):
                if x[i, j] > -math.inf:
                    every.append((s[i] + (x[i, j] - math.log(total)), i, j))
        got = paged.beam(x, s)
        assert len(got) == min(w, len(every))
        best = sorted((-z for z, _, _ in every))[:w]
        np.testing.assert_allclose([-z for z, _, _ in got], best, rtol=1e-12, atol=1e-12)


def test_beam_ties():
    got = paged.beam(np.zeros((2, 3)), np.zeros(2))
    assert [(i, j) for _, i, j in got] == [(0, 0), (0, 1)]
