"""Helpers of the tree tests: seeded problems and their fp64 results."""

from __future__ import annotations

import math
import random

import numpy as np
import torch

from oracle import fp8 as ofp8
from oracle import tree as otree
from paper_2609_19702_amd import binding as B

DEV = "cuda"


def random_parents(rng, n, branch=3):
    kids = [0] * n
    row = [-1]
    for i in range(1, n):
        j = rng.choice([m for m in range(i) if kids[m] < branch])
        kids[j] += 1
        row.append(j)
    return row


class Problem:
    """One call of ``tree_attention``: caches, new tokens and the layout."""

    def __init__(self, batch=2, heads=(4, 4), d=64, prompt=21, grid=(9, 11), nodes=7, bases=None,
                 mode="dense", n_att=1, sinks=0, ring=0, kv="bf16", out="fp32", counts=None,
                 tree=True, branch=3, seed=0, layout="fused", row_base=False, parents=None):
        rng = random.Random(seed)
        self.batch, self.hq, self.hkv, self.d, self.nodes = batch, heads[0], heads[1], d, nodes
        self.prompt, self.sinks = prompt, sinks
        self.length = grid[0] * grid[1]
        self.window = None if mode == "dense" else n_att - sinks
        self.p = B.make_params(prompt, grid[0], grid[1], 1, n_att,
                               B.MODE_DENSE if mode == "dense" else B.MODE_WINDOW, sinks)
        self.s = B.make_shape(batch, heads[0], heads[1], d)
        self.scale = 1 / math.sqrt(d)
        self.bases = list(bases) if bases is not None else [
            rng.randrange(0, max(1, self.length - nodes)) for _ in range(batch)]
        self.counts = counts
        self.ring = ring
        rows = prompt + (ring or self.length)
        g = torch.Generator().manual_seed(seed + 1)
        self.randn = lambda *shape: torch.randn(shape, generator=g)
        hq, hkv = heads
        self.k_scale = self.v_scale = None
        if kv == "fp8":
            self.k, self.v = ((self.randn(batch, hkv, rows, d) * 100).clamp(-448, 448)
                              .to(torch.float8_e4m3fn).to(DEV) for _ in range(2))
            self.k_scale, self.v_scale = ((torch.rand(batch * hkv, generator=g) * 0.02 + 0.005)
                                          .to(DEV) for _ in range(2))
        else:
            self.k, self.v = (self.randn(batch, hkv, rows, d).bfloat16().to(DEV)
                              for _ in range(2))
        if layout == "fused":  # slices of one projection
            x = self.randn(batch, nodes, hq + 2 * hkv, d).bfloat16().to(DEV)
            self.q, self.kn, self.vn = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        elif layout == "heads":  # head-major
            x = self.randn(batch, hq + 2 * hkv, nodes, d).bfloat16().to(DEV).transpose(1, 2)
            self.q, self.kn, self.vn = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        else:  # dense, nodes first: a stride for the batch that is smaller than the node's
            x = self.randn(nodes, batch, hq + 2 * hkv, d).bfloat16().to(DEV).transpose(0, 1)
            self.q, self.kn, self.vn = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        self.parents = parents or [random_parents(rng, nodes, branch) if tree else
                                   otree.chain(nodes) for _ in range(batch)]
        self.tree_plan = None
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        self.base = ints(self.bases)
        self.count = None if counts is None else ints(counts)
        if tree:
            self.parent = ints(self.parents)
            self.tree_plan = torch.empty(B.tree_plan_bytes(batch, nodes), dtype=torch.uint8,
                                         device=DEV)
        self.row_base = None
        if row_base:  # requests in another order than their index
            order = list(range(batch))
            rng.shuffle(order)
            self.order = order
            step = self.k.stride(0)
            self.row_base = torch.tensor([o * step for o in order], dtype=torch.int64, device=DEV)
        else:
            self.order = list(range(batch))
        self.layout = B.kv_layout(self.k, row_base=self.row_base, ring_rows=ring,
                                  k_scale=self.k_scale, v_scale=self.v_scale)
        self.out = torch.full((batch, nodes, hq, d), 7.0, device=DEV,
                              dtype=torch.float32 if out == "fp32" else torch.bfloat16)
        n = B.tree_workspace_bytes(self.p, self.s, nodes)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None
        self.tree = B.make_tree(nodes, self.base, self.count, self.tree_plan)

    def run(self, stream=None):
        if self.tree_plan is not None:
            B.tree_plan(self.parent, self.count, self.tree_plan, stream=stream)
        B.tree_attention(self.p, self.s, self.tree, self.q, self.kn, self.vn, self.k, self.v,
                         self.layout, self.scale, self.out, self.ws, stream=stream)
        return self.out

    def row_of(self, j):
        if self.ring and self.ring < self.length and j >= self.sinks:
            return self.prompt + self.sinks + (j - self.sinks) % (self.ring - self.sinks)
        return self.prompt + j

    def caches64(self):
        """K and V of every request and head as fp64 values."""
        got = []
        for x, sc in ((self.k, self.k_scale), (self.v, self.v_scale)):
            if x.dtype is torch.bfloat16:
                y = x.double().cpu().numpy()
            else:
                y = ofp8.decode_e4m3(x.view(torch.uint8).cpu().numpy())
                if sc is not None:
                    y = y * sc.double().cpu().numpy().reshape(self.batch, self.hkv, 1, 1)
            got.append(y[self.order] if x.dtype is torch.bfloat16 or sc is None else y)
        return got

    def check(self, nodes=None, kv_heads=None):
        """Every node's output against fp64, within the bound of its arithmetic;
        what belongs to no node is as it was."""
        torch.cuda.synchronize()
        out = self.out.double().cpu().numpy()
        k, v = self.caches64()
        q, kn, vn = (x.double().cpu().numpy() for x in (self.q, self.kn, self.vn))
        g = self.hq // self.hkv
        bf16 = self.out.dtype is torch.bfloat16
        worst = 0.0
        for b in range(self.batch):
            n = self.nodes if self.counts is None else min(max(self.counts[b], 0), self.nodes)
            base = min(self.bases[b], self.length)
            if base < -self.prompt:
                n = 0
            assert (out[b, n:] == 7.0).all(), b
            for i in range(n) if nodes is None else [i for i in nodes if i < n]:
                held, up = otree.keys_of(self.parents[b], i, base, self.prompt, self.sinks,
                                         self.window)
                rows = [self.row_of(j) for j in held]
                for h in range(self.hkv) if kv_heads is None else kv_heads:
                    kk = np.concatenate([k[b, h, rows], kn[b, up, h]])
                    vv = np.concatenate([v[b, h, rows], vn[b, up, h]])
                    for e in range(g):
                        ref, band = otree.attend(q[b, i, h * g + e], kk, vv, self.scale)
                        if bf16:  # weights and outputs are rounded to bf16: half a step each
                            band = band + 2 * 2.0 ** -8
                        top = np.abs(vv).max()
                        err = np.abs(out[b, i, h * g + e] - ref).max() / (band * top)
                        worst = max(worst, err)
                        assert err <= 1.0, (b, i, h, e, err, band)
        return worst
