"""A serving loop over pages as the README has it, lengths on the GPU: requests that get
no pages wait, beams that end leave their slots, and every layer's outputs are those of the
rows that each request was given, in bf16 and in fp8 with scales of a layer's own."""

import math

import numpy as np
import pytest
import torch

from oracle import paged as opaged
from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, ints
from tests.test_gpu_pages import e4m3

pytestmark = pytest.mark.gpu


class Serve:
    """Buffers of a loop, and every request's rows in fp64, ``rows[b]`` a list of
    ``(k, v)`` of ``[layers, Hkv, d]``."""

    def __init__(self, batch, pool, kv="bf16", heads=(4, 2), d=64, prompt=13, grid=(6, 6), page=4,
                 layers=2, most=13, seed=0):
        hq, hkv = heads
        self.batch, self.layers, self.hkv, self.d, self.most, self.page = batch, layers, hkv, d, most, page
        self.p = B.make_params(prompt, *grid, 1, 1, B.MODE_DENSE)
        self.s = B.make_shape(batch, hq, hkv, d)
        width = -(-(prompt + grid[0] * grid[1]) // page)
        self.pages = B.make_pages(page, torch.full((batch, width), -1, dtype=torch.int32, device=DEV),
                                  torch.zeros(pool, dtype=torch.int32, device=DEV), ints([0]),
                                  ints([prompt] * batch))
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.k, self.v = (torch.full((layers, pool, hkv, page, d), float("nan"), device=DEV).to(
            torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn) for _ in range(2))
        self.ks = self.vs = None
        if kv == "fp8":
            self.ks, self.vs = (torch.rand((layers, hkv), generator=self.gen, device=DEV) * 0.02 + 0.005
                                for _ in range(2))
        self.all = B.page_layout(self.k[0], self.ks, self.vs)
        self.each = [B.page_layout(self.k[i], *((None, None) if self.ks is None
                                                else (self.ks[i], self.vs[i])))
                     for i in range(layers)]
        self.length = torch.full((batch,), -1, dtype=torch.int32, device=DEV)
        self.slots = torch.zeros((batch, most), dtype=torch.int32, device=DEV)
        self.pos, self.flags = ints([0] * batch), ints([0] * batch)
        self.copies = torch.zeros((batch, 3), dtype=torch.int32, device=DEV)
        self.out = torch.zeros((layers, batch, hq, d), device=DEV)
        n = B.paged_workspace_bytes(self.p, self.s)
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
        self.rows = [[] for _ in range(batch)]

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device=DEV).bfloat16()

    def stored(self, x, scale):
        """The values that a cache holds of rows ``[layers, B, N, Hkv, d]``."""
        if scale is None:
            return x.double().cpu().numpy()
        s = scale[:, None, None, :, None]
        return (e4m3(x.float(), s).float().double() * s.double()).cpu().numpy()

    def step(self, new):
        """The README's lines, then its checks."""
        h = self.hkv
        kv = self.randn(self.layers, self.batch, self.most, 2 * h, self.d)
        q = self.randn(self.layers, self.batch, self.s.num_q_heads, self.d)
        B.page_update(self.p, self.pages, self.length, new, self.slots, self.pos, self.copies, self.flags)
        B.paged_append(self.s, self.slots, kv[:, :, :, :h], kv[:, :, :, h:], self.k, self.v, self.all,
                       self.copies)
        for i in range(self.layers):
            B.paged_attention(self.p, self.s, self.pages, q[i], self.k[i], self.v[i], self.each[i],
                              self.pos, 1 / math.sqrt(self.d), self.out[i], workspace=self.ws)
        given = (self.length >= 0) & (self.flags == 0)
        self.length += torch.where(given, new, 0)
        k, v = self.stored(kv[:, :, :, :h], self.ks), self.stored(kv[:, :, :, h:], self.vs)
        for b, (ok, n) in enumerate(zip(given.tolist(), new.tolist())):
            if ok:
                self.rows[b] += [(k[:, b, i], v[:, b, i]) for i in range(n)]
        self.check(q, given.tolist())

    def check(self, q, given):
        """Lengths are the rows', and outputs theirs in fp64, within the bound of
        ``Attend.check``."""
        assert [max(x, 0) for x in self.length.tolist()] == [len(x) for x in self.rows]
        out, q = self.out.double().cpu().numpy(), q.double().cpu().numpy()
        g, front = self.s.num_q_heads // self.hkv, self.pages.prompt.tolist()
        scale, u = 1 / math.sqrt(self.d), 2.0 ** -24
        for b, rows in enumerate(self.rows):
            if not given[b] or len(rows) <= front[b]:
                assert (out[:, b] == 0).all() and self.pos[b] == -1
                continue
            assert self.pos[b] == len(rows) - 1 - front[b]
            k, v = (np.stack([r[i] for r in rows]) for i in range(2))  # [n, layers, Hkv, d]
            for i in range(self.layers):
                for hq in range(self.s.num_q_heads):
                    kh, vh, qh = k[:, i, hq // g], v[:, i, hq // g], q[i, b, hq]
                    want, _, mass = opaged.attention(qh, kh, vh, scale)
                    dz = (np.abs(kh) @ np.abs(qh)).max() * scale * (self.d + 4) * u
                    rel = 2 * dz + 4 * u + (2 * len(rows) + 64) * u
                    assert (np.abs(out[i, b, hq] - want) <= rel * mass + u * np.abs(want)).all()

    def reorder(self, parent):
        """The README's lines after a choice of beams."""
        B.page_reorder(self.pages, parent)
        self.length.copy_(torch.where(parent >= 0, self.length[parent.clamp(min=0)], -1))
        self.rows = [list(self.rows[p]) if p >= 0 else [] for p in parent.tolist()]

    def users(self):
        n = torch.zeros_like(self.pages.refs)
        at = self.pages.table[self.pages.table >= 0].long()
        return n.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_requests_that_get_no_pages_wait(kv):
    """Four requests in a pool for less than three, one slot never used: who gets nothing
    holds what it held, and goes on when others have left."""
    x = Serve(5, pool=20, kv=kv)
    one = torch.ones(5, dtype=torch.int32, device=DEV)
    x.length[:4] = 0
    waited = finished = 0
    for _ in range(120):
        first = x.length == 0
        x.step(torch.where(first, 13, one))
        flags = x.flags.tolist()
        waited += sum(flags)
        done = x.length >= 13 + 20
        finished += int(done.sum())
        held = [b for b, n in enumerate(x.length.tolist()) if n > 0]
        if held and all(flags[b] for b in held):  # they wait for each other: the last gives up
            done[held[-1]] = True
        x.length.masked_fill_(done, -1)
        x.rows = [[] if d else r for d, r in zip(done.tolist(), x.rows)]
        back = (x.length < 0) & (torch.arange(5, device=DEV) < 4) & ~done
        x.length.masked_fill_(back, 0)
        assert torch.equal(x.users(), x.pages.refs) and x.length[4] == -1
    assert waited > 10 and finished > 5


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_beams_that_end(kv):
    """Steps with fewer candidates than beams: the others' slots are unused, without rows or
    pages, until a later choice fills them again."""
    groups, w, vocab = 2, 4, 50
    x = Serve(groups * w, pool=110, kv=kv)
    score, parent, token = (torch.zeros((groups, w), dtype=t, device=DEV)
                            for t in (torch.float32, torch.int32, torch.int32))
    score[:, 1:] = -math.inf
    ws = torch.empty(B.beam_workspace_bytes(groups, w, vocab), dtype=torch.uint8, device=DEV)
    x.length[::w] = 0
    x.step(ints([13] * groups * w))
    one, ended, copied = ints([1] * groups * w), 0, 0
    for i in range(24):
        z = torch.randn((groups, w, vocab), generator=x.gen, device=DEV)
        if i % 5 == 3:  # the first request goes on from one beam alone, the second from two
            live = [(score[g] > -math.inf).nonzero().view(-1).tolist() for g in range(groups)]
            z[:, :, 1:] = -math.inf
            for g in range(groups):
                z[g, live[g][-1 - g]:, 0] = 0.5
                z[g, :live[g][-1 - g], 0] = -math.inf
        B.beam_select(z, score, score, parent, token, ws)
        x.reorder(parent.view(-1))
        gone = (parent.view(-1) < 0).tolist()
        ended += sum(gone)
        x.step(one)
        copied += int((x.copies[:, 0] >= 0).sum())
        assert x.flags.tolist() == [0] * groups * w
        assert torch.equal(x.users(), x.pages.refs)
        for b, g in enumerate(gone):
            if g:
                assert x.length[b] == -1 and (x.pages.table[b] == -1).all()
                assert (x.slots[b] == -1).all() and score.view(-1)[b] == -math.inf
    assert ended == 5 * 5 and copied > 5
