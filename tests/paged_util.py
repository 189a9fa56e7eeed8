"""Helpers of the tests of paged caches: seeded problems and their fp64 results."""

from __future__ import annotations

import math
import random

import numpy as np
import torch

from oracle import paged as opaged
from paper_2609_19702_amd import binding as B

DEV = "cuda"
MODES = {"dense": B.MODE_DENSE, "diagonal": B.MODE_DIAGONAL, "window": B.MODE_WINDOW}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Attend:
    """One call of ``paged_attention``.  Every row of the pool that no request
    attends holds ``hidden`` in K and V."""

    def __init__(self, batch=2, heads=(4, 4), d=64, prompt=21, grid=(9, 11), page=16, pos=None,
                 mode="dense", n_att=1, sinks=0, window=1, kv="bf16", out="fp32", prompts=None,
                 seed=0, hidden=float("nan"), holes=0.0, spare=3, order="page", scale=None,
                 scales=True, logits=True, width=None):
        rng = self.rng = random.Random(seed)
        self.batch, self.hq, self.hkv, self.d, self.page = batch, heads[0], heads[1], d, page
        self.mode, self.n_att, self.sinks, self.length = mode, n_att, sinks, grid[0] * grid[1]
        self.p = B.make_params(prompt, grid[0], grid[1], window, n_att, MODES[mode], sinks)
        self.s = B.make_shape(batch, heads[0], heads[1], d)
        self.scale = 1 / math.sqrt(d) if scale is None else scale
        self.pos = list(pos) if pos is not None else [rng.randrange(self.length)
                                                      for _ in range(batch)]
        self.prompts = list(prompts) if prompts is not None else [prompt] * batch
        front = [min(max(x, 0), prompt) for x in self.prompts]
        width = width or -(-(prompt + self.length) // page)
        pool = batch * width + spare
        pages = list(range(pool))
        rng.shuffle(pages)
        self.table = [[-1] * width for _ in range(batch)]
        self.rows = []  # [b][h]: attended rows, those without a page as None
        kept = self.kept = [[None] * self.hkv for _ in range(batch)]
        used = {}
        for b in range(batch):
            t = min(self.pos[b], self.length - 1)
            heads_rows = []
            for h in range(self.hkv):
                if t >= 0 and mode == "diagonal":
                    kept[b][h] = self.random_kept(t, window)
                at = [] if t < 0 else list(range(front[b])) + [
                    front[b] + j for j in opaged.attended_positions(mode, t, n_att, sinks,
                                                                    kept[b][h])]
                heads_rows.append(at)
            for i in sorted({r // page for at in heads_rows for r in at}):
                if i < width and rng.random() >= holes:
                    self.table[b][i] = pages.pop()
            self.rows.append([[r if r // page < width and self.table[b][r // page] >= 0 else None
                               for r in at] for at in heads_rows])
            for h, at in enumerate(self.rows[b]):
                for r in at:
                    if r is not None:
                        used.setdefault((self.table[b][r // page], h), []).append(r % page)
        g = torch.Generator().manual_seed(seed + 1)
        shape = (pool, self.hkv, page, d)
        self.k, self.v = torch.full(shape, hidden), torch.full(shape, hidden)
        for x in (self.k, self.v):
            for (gpage, h), at in used.items():
                at = sorted(set(at))
                x[gpage, h, at] = torch.randn((len(at), d), generator=g)
        self.k_scale = self.v_scale = None
        if kv == "fp8":
            if scales:
                self.k_scale, self.v_scale = (torch.rand(self.hkv, generator=g).to(DEV) * 0.02 + 0.005
                                              for _ in range(2))
            mul = 100 if scales else 1
            self.k, self.v = ((x * mul).clamp(-448, 448).to(torch.float8_e4m3fn)
                              for x in (self.k, self.v))
        else:
            self.k, self.v = self.k.bfloat16(), self.v.bfloat16()
        self.k64, self.v64 = (x.float().double().numpy() for x in (self.k, self.v))
        if kv == "fp8" and scales:
            self.k64, self.v64 = (x * y.double().cpu().numpy()[None, :, None, None]
                                  for x, y in ((self.k64, self.k_scale), (self.v64, self.v_scale)))
        self.k, self.v = (self.placed(x, order) for x in (self.k, self.v))
        self.q = torch.randn((batch, self.hq, d), generator=g).bfloat16().to(DEV)
        self.pages = B.make_pages(page, ints(self.table),
                                  prompt=ints(self.prompts) if prompts is not None else None)
        self.layout = B.page_layout(self.k, self.k_scale, self.v_scale)
        self.pos_t = ints(self.pos)
        self.out = torch.full((batch, self.hq, d), 7.0, device=DEV,
                              dtype=torch.float32 if out == "fp32" else torch.bfloat16)
        n = B.paged_workspace_bytes(self.p, self.s)
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None
        self.plan = self.logits = None
        if mode == "diagonal":
            self.plan = torch.zeros(B.plan_bytes(self.p, self.s), dtype=torch.uint8, device=DEV)
            count, _, places = B.plan_views(self.p, self.s, self.plan)
            for b in range(batch):
                for h in range(self.hkv):
                    line = kept[b][h] or []
                    count[b * self.hkv + h] = len(line)
                    places[b * self.hkv + h, :len(line)] = ints(line)
            if logits:
                self.cap = places.shape[1]
                self.logits = torch.full((batch, self.hq, self.cap), 7.0, device=DEV)

    def random_kept(self, t, window):
        """The sinks, ``t`` and random positions of the window, in order."""
        n = min(t + 1, self.n_att)
        front = list(range(min(self.sinks, t + 1)))
        if len(front) == n:
            return front
        rest = list(range(max(self.sinks, t - window + 1), t))
        return front + sorted(self.rng.sample(rest, n - len(front) - 1)) + [t]

    @staticmethod
    def placed(x, order):
        """The same values in another order of memory."""
        if order == "page":
            return x.to(DEV)
        if order == "head":  # heads outermost
            return x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
        if order == "row":  # rows before heads, and rows and pages apart
            n, h, p, d = x.shape
            y = torch.full((n, p + 1, h + 2, d + 32), float("nan")).to(x.dtype).to(DEV)
            y[:, :p, :h, :d].copy_(x.transpose(1, 2))
            return y[:, :p, :h, :d].transpose(1, 2)
        raise ValueError(order)

    def run(self, stream=None):
        B.paged_attention(self.p, self.s, self.pages, self.q, self.k, self.v, self.layout,
                          self.pos_t, self.scale, self.out, self.plan, self.logits, self.ws,
                          stream=stream)
        return self.out

    def check(self, requests=None, kv_heads=None):
        """Outputs and logits against fp64.  The bound counts the roundings: a score
        is a sum of d exact products in fp32 and two products more; a weight moves
        by twice the largest error of a score and by its exponential's (two units);
        the sums over n rows round n times, a tile of 32 rows once more, weights
        of bf16 outputs are off by 2^-18, and the output is rounded once."""
        u = 2.0 ** -24
        out, q = self.out.double().cpu().numpy(), self.q.double().cpu().numpy()
        logits = None if self.logits is None else self.logits.double().cpu().numpy()
        group = self.hq // self.hkv
        for b in range(self.batch) if requests is None else requests:
            t = min(self.pos[b], self.length - 1)
            for h in range(self.hkv) if kv_heads is None else kv_heads:
                at = self.rows[b][h]
                there = [r for r in at if r is not None]
                page = [self.table[b][r // self.page] for r in there]
                off = [r % self.page for r in there]
                k, v = self.k64[page, h, off], self.v64[page, h, off]
                for hq in range(h * group, (h + 1) * group):
                    want, z, mass = opaged.attention(q[b, hq], k, v, self.scale)
                    dz = np.abs(k) @ np.abs(q[b, hq]) * abs(self.scale) * (self.d + 4) * u
                    n = len(there)
                    rel = 2 * (dz.max() if n else 0) + 4 * u + (2 * n + 64) * u
                    half = torch.finfo(self.out.dtype).eps / 2
                    if self.out.dtype == torch.bfloat16:
                        rel += 2.0 ** -17
                    bound = rel * mass + half * np.abs(want) + 1e-30
                    err = np.abs(out[b, hq] - want)
                    assert (err <= bound).all(), (b, hq, n, (err / bound).max())
                    if logits is None:
                        continue
                    front = len(at) - len(self.kept[b][h] or [])
                    line = logits[b, hq]
                    assert (line[len(at) - front:] == 7.0).all()
                    i = 0
                    for e, r in enumerate(at):
                        if e >= front:
                            if r is None:
                                assert line[e - front] == -math.inf
                            else:
                                assert abs(line[e - front] - z[i]) <= dz[i] + 1e-30
                        i += r is not None
