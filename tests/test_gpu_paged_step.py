"""The calls over pages together, as a serving loop issues them: prompts in, steps of
Algorithm 1 over pages against the same steps over a linear cache, several images of
one prompt, beams, requests that come and go."""

import math
import random

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, MODES, ints

pytestmark = pytest.mark.gpu


class Loop:
    """A batch over pages and, beside it, what its rows are in a linear cache."""

    def __init__(self, batch, heads, d, prompt, grid, page, mode, window=1, n_att=1, sinks=0,
                 pool=None, seed=0):
        hq, self.hkv = heads
        self.batch, self.d, self.prompt, self.page = batch, d, prompt, page
        self.length = grid[0] * grid[1]
        self.p = B.make_params(prompt, grid[0], grid[1], window, n_att, MODES[mode], sinks)
        self.s = B.make_shape(batch, hq, self.hkv, d)
        width = -(-(prompt + self.length) // page)
        pool = pool or batch * width
        self.pages = B.make_pages(page, torch.full((batch, width), -1, dtype=torch.int32, device=DEV),
                                  torch.zeros(pool, dtype=torch.int32, device=DEV), ints([0]))
        self.k, self.v = (torch.full((pool, self.hkv, page, d), float("nan"), device=DEV).bfloat16()
                          for _ in range(2))
        self.layout = B.page_layout(self.k)
        self.lin = [torch.zeros((batch, self.hkv, prompt + self.length, d), device=DEV).bfloat16()
                    for _ in range(2)]
        self.pos, self.flags = ints([-1] * batch), ints([0] * batch)
        self.copies = torch.full((batch, 3), -1, dtype=torch.int32, device=DEV)
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.scale = 1 / math.sqrt(d)
        self.out = torch.zeros((batch, hq, d), device=DEV)
        n = B.paged_workspace_bytes(self.p, self.s)
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
        self.bufs = B.alloc_buffers(self.p, self.s)
        self.lin_bufs = B.alloc_buffers(self.p, self.s)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device=DEV).bfloat16()

    def rows_in(self, lengths, new, most):
        """Random new rows into the pages and into the linear cache."""
        slots = torch.zeros((self.batch, most), dtype=torch.int32, device=DEV)
        B.page_update(self.p, self.pages, ints(lengths), ints(new), slots, self.pos, self.copies,
                      self.flags)
        rows = self.randn(self.batch, most, 2 * self.hkv, self.d)
        B.paged_append(self.s, slots, rows[:, :, :self.hkv], rows[:, :, self.hkv:], self.k, self.v,
                       self.layout, self.copies)
        for b, (at, n) in enumerate(zip(lengths, new)):
            if at >= 0 and n:
                self.lin[0][b, :, at:at + n] = rows[b, :n, :self.hkv].transpose(0, 1)
                self.lin[1][b, :, at:at + n] = rows[b, :n, self.hkv:].transpose(0, 1)
        return rows

    def step(self):
        """One decode step of both, and that they agree: each output is within its bound
        of the exact one (2e-5 of the largest here: scores of a few units, sums of
        some hundred rows), so both are within twice that of each other."""
        q = self.randn(self.batch, self.s.num_q_heads, self.d)
        diagonal = self.p.mode == B.MODE_DIAGONAL
        if diagonal:
            B.plan(self.p, self.s, self.pos, self.bufs.state, self.bufs.plan)
        B.paged_attention(self.p, self.s, self.pages, q, self.k, self.v, self.layout, self.pos,
                          self.scale, self.out, self.bufs.plan if diagonal else None,
                          self.bufs.logits if diagonal else None, self.ws)
        if diagonal:
            B.select(self.p, self.s, self.pos, self.bufs.plan, self.bufs.logits, self.bufs.state)
        lin = self.lin_bufs
        B.decode_step(self.p, self.s, q, *self.lin, B.kv_layout(self.lin[0]), self.pos, lin.state,
                      lin.plan, self.scale, lin.out, lin.logits, lin.workspace)
        assert (self.out - lin.out).abs().max() <= 4e-5 * lin.out.abs().max()
        if diagonal:
            ours, theirs = (B.state_views(self.p, self.s, x.state) for x in (self.bufs, lin))
            assert torch.equal(ours[0], theirs[0]) and torch.equal(ours[2], theirs[2])


@pytest.mark.parametrize("heads,d", [((4, 4), 64), ((8, 2), 128)])
@pytest.mark.parametrize("mode,sinks", [("dense", 0), ("window", 4), ("diagonal", 0), ("diagonal", 4)])
def test_images_over_pages(heads, d, mode, sinks):
    """Whole images of requests that begin at different steps.  Pages behind the window
    go back, so the window modes live in a pool of half the rows."""
    prompt, grid, page = 21, (10, 10), 8
    batch = 3
    rows = -(-(prompt + 100) // page) * batch
    x = Loop(batch, heads, d, prompt, grid, page, mode, window=40, n_att=20, sinks=sinks,
             pool=rows if mode == "dense" else rows * 2 // 3)
    B.state_reset(x.p, x.s, x.bufs.state)
    B.state_reset(x.p, x.s, x.lin_bufs.state)
    begin = [0, 7, 13]
    for t in range(113):
        lengths, new = [], []
        for b in range(batch):
            at = t - begin[b]
            lengths.append(-1 if at < 0 or at >= 100 else 0 if at == 0 else prompt + at)
            new.append(prompt + 1 if at == 0 else int(0 < at < 100))
        x.rows_in(lengths, new, prompt + 1)
        assert x.flags.tolist() == [0] * batch
        assert x.pos.tolist() == [t - s if 0 <= t - s < 100 else -1 for s in begin]
        x.step()


def test_several_images_of_one_prompt():
    """They share its whole pages; the one that it ends in is copied."""
    x = Loop(4, (4, 4), 64, 21, (6, 6), 8, "dense", pool=40)
    x.rows_in([0, -1, -1, -1], [21, 0, 0, 0], 21)
    B.page_reorder(x.pages, ints([0, 0, 0, 0]))
    for t in x.lin:
        t[1:] = t[:1]
    for i in range(30):
        x.rows_in([21 + i] * 4, [1] * 4, 1)
        x.step()
        if i == 0:
            assert (x.pages.refs == 4).sum() == 2 and (x.copies[:, 2] == 5).all()
    assert (x.pages.refs > 0).sum() == 2 + 4 * (-(-51 // 8) - 2)
    x.rows_in([-1] * 4, [0] * 4, 1)
    assert (x.pages.refs == 0).all() and (x.pages.table == -1).all()


def test_beams_over_pages():
    """A beam search: choice, reorder, update, append, attention; the linear cache moves
    its rows instead."""
    groups, w, vocab, prompt = 2, 3, 700, 13
    batch = groups * w
    x = Loop(batch, (4, 2), 64, prompt, (6, 6), 4, "dense", pool=90)
    B_ = lambda dtype: torch.zeros((groups, w), dtype=dtype, device=DEV)  # noqa: E731
    score, parent, token = B_(torch.float32), B_(torch.int32), B_(torch.int32)
    score[:, 1:] = -math.inf  # all beams of a prompt begin as one
    ws = torch.empty(B.beam_workspace_bytes(groups, w, vocab), dtype=torch.uint8, device=DEV)
    first = [0 if b % w == 0 else -1 for b in range(batch)]
    x.rows_in(first, [prompt] * batch, prompt)
    moved = 0
    for i in range(25):
        z = torch.randn((groups, w, vocab), generator=x.gen, device=DEV)
        B.beam_select(z, score, score, parent, token, ws)
        B.page_reorder(x.pages, parent.view(-1))
        at = parent.view(-1).long()
        x.lin = [t[at].contiguous() for t in x.lin]
        x.rows_in([prompt + i] * batch, [1] * batch, 1)
        assert x.flags.tolist() == [0] * batch
        x.step()
        moved += int((x.copies[:, 0] >= 0).sum())
        n = torch.zeros_like(x.pages.refs)
        used = x.pages.table[x.pages.table >= 0].long()
        assert torch.equal(n.index_add_(0, used, torch.ones_like(used, dtype=torch.int32)),
                           x.pages.refs)
    assert moved > 5


def test_a_prompt_through_tree_attention():
    """Its attention needs no cache; then its rows go into pages, and the first step
    attends them as after kv_append."""
    x = Loop(2, (8, 2), 128, 37, (6, 6), 16, "dense")
    rows = x.rows_in([0, 0], [37, 37], 37)
    tree = B.make_tree(37, ints([-37, -37]))
    q, out = x.randn(2, 37, 8, 128), torch.zeros((2, 37, 8, 128), device=DEV)
    n = B.tree_workspace_bytes(x.p, x.s, 37)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    outs = []
    for k, v, layout in ((*x.lin, B.kv_layout(x.lin[0])),
                         (x.k, x.v, B.kv_layout(x.k, row_base=torch.zeros(2, dtype=torch.int64,
                                                                         device=DEV)))):
        B.tree_attention(x.p, x.s, tree, q, rows[:, :, :2], rows[:, :, 2:], k, v, layout, x.scale,
                         out, ws)
        outs.append(out.clone())
    assert torch.equal(*outs)
    lin = [torch.zeros_like(t) for t in x.lin]
    B.kv_append(x.p, x.s, tree, rows[:, :, :2], rows[:, :, 2:], *lin, B.kv_layout(lin[0]))
    assert all(torch.equal(p, q) for p, q in zip(lin, x.lin))
    x.rows_in([37, 37], [1, 1], 1)
    x.step()


def test_a_captured_step():
    """Update, append and attention of a step in one graph, lengths advanced in it."""
    x = Loop(3, (4, 4), 64, 9, (8, 8), 8, "window", n_att=20, sinks=2, pool=24)
    x.rows_in([0, 0, 0], [9, 9, 9], 9)
    length, slots = ints([9, 9, 9]), ints([[-1]] * 3)
    rows, q = x.randn(3, 1, 8, 64), x.randn(3, 4, 64)

    def issue():
        B.page_update(x.p, x.pages, length, None, slots, x.pos, x.copies, x.flags)
        B.paged_append(x.s, slots, rows[:, :, :4], rows[:, :, 4:], x.k, x.v, x.layout, x.copies)
        B.paged_attention(x.p, x.s, x.pages, q, x.k, x.v, x.layout, x.pos, x.scale, x.out,
                          workspace=x.ws)
        length.add_(1)

    issue()
    x.lin[0][:, :, 9], x.lin[1][:, :, 9] = rows[:, 0, :4], rows[:, 0, 4:]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        issue()
    lin = x.lin_bufs
    for i in range(10, 60):
        rows.copy_(x.randn(3, 1, 8, 64))
        q.copy_(x.randn(3, 4, 64))
        g.replay()
        x.lin[0][:, :, i], x.lin[1][:, :, i] = rows[:, 0, :4], rows[:, 0, 4:]
        assert x.pos.tolist() == [i - 9] * 3 and x.flags.tolist() == [0] * 3
        B.decode_step(x.p, x.s, q, *x.lin, B.kv_layout(x.lin[0]), x.pos, lin.state, lin.plan,
                      x.scale, lin.out, lin.logits, lin.workspace)
        assert (x.out - lin.out).abs().max() <= 4e-5 * lin.out.abs().max()


def test_requests_come_and_go():
    rng = random.Random(1)
    x = Loop(5, (4, 2), 64, 11, (5, 5), 4, "dense", pool=30)
    at = [-1] * 5
    for _ in range(60):
        new = []
        for b in range(5):
            if at[b] < 0 or at[b] >= 36 or rng.random() < 0.03:
                at[b] = rng.choice([-1, 0])
            new.append(11 if at[b] == 0 else 1 if at[b] > 0 else 0)
        x.rows_in(at, new, 11)
        short = x.flags.tolist()
        x.pos.copy_(torch.where(ints(at) == 0, -1, x.pos))  # prompts have no token to decode yet
        x.step()
        at = [-1 if f else a + n if a >= 0 else -1 for a, n, f in zip(at, new, short)]
