"""The choice of beams against fp64, ties and what is no candidate."""

import math

import numpy as np
import pytest
import torch

from oracle import paged as opaged
from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


class Beam:
    def __init__(self, x, score):
        self.x, self.score = x, score
        b, w, v = x.shape
        self.next = torch.full((b, w), 7.0, device=DEV)
        self.parent = torch.full((b, w), 7, dtype=torch.int32, device=DEV)
        self.token = torch.full((b, w), 7, dtype=torch.int32, device=DEV)
        self.ws = torch.full((B.beam_workspace_bytes(b, w, v),), 255, dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        B.beam_select(self.x, self.score, self.next, self.parent, self.token, self.ws, stream=stream)
        return self

    def check(self):
        """Choices equal; a score is off by its own rounding and by that of the log of
        the sum: an exponential by two units of 2^-24 and by its argument's rounding,
        whose mean over the terms is at most log2(e) log V."""
        b, w, v = self.x.shape
        x, s = self.x.double().cpu().numpy(), self.score.double().cpu().numpy()
        nxt, parent, token = (t.cpu().numpy() for t in (self.next, self.parent, self.token))
        off = (4 + 2 * math.log2(v + 1)) * 2.0 ** -24
        for i in range(b):
            want = opaged.beam(x[i], s[i])
            for k in range(w):
                if k >= len(want):
                    assert (nxt[i, k], parent[i, k], token[i, k]) == (-INF, -1, -1)
                    continue
                z, pw, pv = want[k]
                assert (parent[i, k], token[i, k]) == (i * w + pw, pv), (i, k)
                assert abs(nxt[i, k] - z) <= off + abs(z) * 2.0 ** -24
        return self


def logits(b, w, v, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((b, w, v), generator=g)
    return x.to(dtype).to(DEV), (-20 * torch.rand((b, w), generator=g)).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("w", [1, 2, 3, 4, 5, 8, 16])
def test_beams(dtype, w):
    for i, (b, v) in enumerate(((1, 16384), (3, 5003), (2, 1), (2, 7), (5, 2048), (3, 2049), (1, 255),
                                (2, 65539))):
        Beam(*logits(b, w, v, dtype, 100 * w + i)).run().check()


def test_a_large_vocabulary_and_many_requests():
    Beam(*logits(1, 4, 1 << 20, torch.bfloat16, 1)).run().check()
    Beam(*logits(300, 4, 1000, torch.float32, 2)).run().check()
    Beam(*logits(40, 16, 9000, torch.bfloat16, 3)).run().check()


def test_ties_go_to_the_lowest_place():
    for w, v in ((4, 5000), (8, 3), (3, 40000)):
        x = torch.zeros((2, w, v), device=DEV)
        Beam(x, torch.full((2, w), -3.0, device=DEV)).run().check()
        x = torch.randint(0, 2, (2, 1, v), device=DEV).float().expand(2, w, v).contiguous()
        Beam(x.bfloat16(), torch.full((2, w), -3.0, device=DEV)).run().check()
    x = torch.zeros((1, 2, 600), device=DEV)
    x[0, 0, ::2] = -0.0
    y = Beam(x, torch.zeros((1, 2), device=DEV)).run().check()
    assert y.token.tolist() == [[0, 1]] and y.parent.tolist() == [[0, 0]]


def test_beams_that_have_not_begun_or_are_finished():
    x, s = logits(3, 4, 3000, torch.float32, 1)
    s[:, 1:] = -INF
    y = Beam(x, s).run().check()
    assert set(y.parent[2].tolist()) == {8}
    x[0, 1:] = -INF  # finished: one token left, at no cost
    x[0, 1:, 17] = 3.0
    s[0] = torch.tensor([-1.0, -0.5, -90.0, -0.5])
    y = Beam(x, s).run().check()
    assert y.token[0, 0] == 17 and y.next[0, 0] == -0.5 and y.parent[0, 1] == 3


def test_fewer_candidates_than_beams():
    x = torch.full((2, 4, 5), -INF, device=DEV)
    x[0, 2, 3], x[0, 1, 0] = 1.0, 2.0
    y = Beam(x, torch.zeros((2, 4), device=DEV)).run().check()
    assert y.parent.tolist() == [[1, 2, -1, -1], [-1] * 4]


@pytest.mark.parametrize("bad", [NAN, INF])
def test_rows_without_a_distribution_are_no_candidates(bad):
    for dtype in (torch.float32, torch.bfloat16):
        x, s = logits(2, 4, 9001, dtype, 5)
        x[0, 1, 9000], x[1, 3, 0] = bad, bad
        y = Beam(x, s).run().check()
        assert 1 not in y.parent[0].tolist() and 7 not in y.parent[1].tolist()
    x, s = logits(1, 2, 300, torch.float32, 5)
    s[0, 0] = NAN
    y = Beam(x, s).run().check()
    assert y.parent.tolist() == [[1, 1]]


def test_large_logits_and_far_scores():
    x, s = logits(2, 4, 4000, torch.float32, 6, spread=1e4)
    Beam(x, s).run().check()
    Beam(x * 1e33, s).run()
    x, s = logits(2, 4, 4000, torch.float32, 6)
    y = Beam(x, s * 1e6).run()
    want = [opaged.beam(a, b) for a, b in zip(x.double().cpu().numpy(),
                                              (s * 1e6).double().cpu().numpy())]
    assert y.token.tolist() == [[c[2] for c in line] for line in want]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_apart_and_unaligned(dtype):
    whole, s = logits(3, 4, 3011, dtype, 7)
    for lo, hi in ((0, 3000), (1, 3011), (3, 2050), (5, 6)):
        x = whole[:, :, lo:hi]
        Beam(x, s).run().check()
    Beam(whole[:, :1], s[:, :1].contiguous()).run().check()
    Beam(whole[1:2], s[1:2]).run().check()


def test_scores_in_place():
    x, s = logits(2, 4, 3000, torch.float32, 8)
    want = Beam(x, s.clone()).run().check()
    y = Beam(x, s)
    y.next = s
    y.run()
    assert torch.equal(s, want.next) and torch.equal(y.parent, want.parent)


def test_graph_and_streams():
    a, b = Beam(*logits(2, 4, 9000, torch.float32, 9)), Beam(*logits(4, 8, 3000, torch.bfloat16, 10))
    want = []
    for x in (a, b):
        x.run().check()
        want.append([t.clone() for t in (x.next, x.parent, x.token)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for x, st in zip((a, b), streams):
            x.run(stream=st)
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        assert all(torch.equal(p, q) for p, q in zip((x.next, x.parent, x.token), w))
    ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device=DEV)
    graphs = []
    for x in (a, b):
        x.ws = ws
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for i in (0, 1, 1, 0):
        ws.fill_(255)
        for x in (a, b):
            x.next.fill_(7.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal((a, b)[i].next, want[i][0])
    assert np.isfinite(want[0][0].cpu().numpy()).all()
