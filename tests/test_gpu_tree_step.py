"""The tree calls together, as a program uses them: a prompt and an image's
first tokens on their way into a cache in chunks, and speculative decoding
against token-by-token decoding."""

import math
import random

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2609_19702_amd import binding as B
from tests.gpu_util import DEV
from tests.tree_util import random_parents

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("mode", ["dense", "ring"])
def test_chunks_fill_a_cache(kv, mode):
    """Two requests of one length, in chunks of different sizes (the first of the
    prompt, one across its end): the caches are those of the whole sequence, and
    every chunk attends what it would in one call."""
    batch, hq, hkv, d, lp, grid = 2, 8, 4, 64, 19, (6, 8)
    length, total = 48, 19 + 45
    g = torch.Generator().manual_seed(3)
    x = torch.randn((batch, total, hq + 2 * hkv, d), generator=g).bfloat16().to(DEV)
    q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    if mode == "dense":
        p, ring = B.make_params(lp, *grid, 1, 1, B.MODE_DENSE), 0
        sinks, window = 0, None
    else:
        p, ring = B.make_params(lp, *grid, 1, 14, B.MODE_WINDOW, 3), 16
        sinks, window = 3, 11
    s = B.make_shape(batch, hq, hkv, d)
    rows = lp + (ring or length)
    scales = [None, None]
    if kv == "fp8":
        kc, vc = (torch.zeros((batch, hkv, rows, d), dtype=torch.uint8, device=DEV)
                  for _ in range(2))
        scales = [torch.full((batch * hkv,), 0.02, device=DEV) for _ in range(2)]
    else:
        kc, vc = (torch.zeros((batch, hkv, rows, d), dtype=torch.bfloat16, device=DEV)
                  for _ in range(2))
    lay = B.kv_layout(kc, ring_rows=ring, k_scale=scales[0], v_scale=scales[1])
    scale, at = 1 / math.sqrt(d), 0
    outs = []
    for n in (7, 5, 20, 1, 31):
        tree = B.make_tree(n, ints([at - lp] * batch))
        part = slice(at, at + n)
        out = torch.empty((batch, n, hq, d), device=DEV)
        ws = torch.empty(max(1, B.tree_workspace_bytes(p, s, n)), dtype=torch.uint8, device=DEV)
        B.tree_attention(p, s, tree, q[:, part], k[:, part], v[:, part], kc, vc, lay, scale, out, ws)
        B.kv_append(p, s, tree, k[:, part], v[:, part], kc, vc, lay)
        outs.append(out)
        at += n
    assert at == total
    # the caches: the last token of every row
    code = lambda y, sc: y if kv == "bf16" else torch.from_numpy(
        otree.encode_e4m3((y.float() / sc).cpu().numpy())).to(DEV)
    for cache, new, sc in ((kc, k, 0.02), (vc, v, 0.02)):
        want = torch.zeros_like(cache)
        for t in range(total):
            j = t - lp
            r = t if not ring or j < sinks else lp + sinks + (j - sinks) % (ring - sinks)
            want[:, :, r] = code(new[:, t], sc)
        assert torch.equal(cache.view(torch.uint8), want.view(torch.uint8))
    # the outputs: within their bound of fp64, over the rows as the cache holds them
    out = torch.cat(outs, 1).double().cpu().numpy()
    chunk_of = sum(([i] * n for i, n in enumerate((7, 5, 20, 1, 31))), [])
    starts = np.cumsum([0, 7, 5, 20, 1, 31])
    kn, vn, qn = (y.double().cpu().numpy() for y in (k, v, q))
    old = []
    for y in (k, v):
        z = y.float().cpu().numpy()
        if kv == "fp8":
            from oracle import fp8 as ofp8
            sc = np.float32(0.02)
            z = ofp8.decode_e4m3(otree.encode_e4m3(z / sc)) * float(sc)
        old.append(z.astype(np.float64))
    for b in range(batch):
        for t in range(total):
            first = starts[chunk_of[t]]
            see = [u for u in range(t + 1)
                   if otree.reach(t - lp, u - lp, sinks, window)]
            for h in range(hkv):
                kk = np.stack([(old[0] if u < first else kn)[b, u, h] for u in see])
                vv = np.stack([(old[1] if u < first else vn)[b, u, h] for u in see])
                for e in range(hq // hkv):
                    ref, band = otree.attend(qn[b, t, h * (hq // hkv) + e], kk, vv, scale)
                    err = np.abs(out[b, t, h * (hq // hkv) + e] - ref).max()
                    assert err <= band * np.abs(vv).max(), (b, t, h, e)


class Toy:
    """Two layers of attention over random weights; ``heads`` of 64."""

    def __init__(self, batch, vocab=53, hq=4, hkv=2, prompt=9, grid=(5, 8), seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *n: torch.randn(n, generator=g).to(DEV)
        self.d, self.hq, self.hkv, self.vocab, self.batch = 64, hq, hkv, vocab, batch
        dim = hq * 64
        self.emb, self.head = r(vocab, dim), r(dim, vocab) / math.sqrt(dim)
        self.w = [r(dim, (hq + 2 * hkv) * 64) / math.sqrt(dim) for _ in range(2)]
        self.prompt, self.length = prompt, grid[0] * grid[1]
        self.p = B.make_params(prompt, *grid, 1, 1, B.MODE_DENSE)
        self.s = B.make_shape(batch, hq, hkv, 64)
        rows = prompt + self.length
        self.k, self.v = (torch.zeros((2, batch, hkv, rows, 64), dtype=torch.bfloat16, device=DEV)
                          for _ in range(2))
        self.lay = B.kv_layout(self.k[0])

    def forward(self, tokens, tree):
        """Logits of every node, and the K and V rows of both layers."""
        b, n = tokens.shape
        x = self.emb[tokens.long()]
        new = []
        for i in range(2):
            y = (x @ self.w[i]).bfloat16().view(b, n, self.hq + 2 * self.hkv, 64)
            q, k, v = y.split([self.hq, self.hkv, self.hkv], 2)
            out = torch.zeros((b, n, self.hq, 64), device=DEV)
            size = B.tree_workspace_bytes(self.p, self.s, n)
            ws = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None
            B.tree_attention(self.p, self.s, tree, q, k, v, self.k[i], self.v[i], self.lay, 0.125,
                             out, ws)
            x = x + out.reshape(b, n, -1)
            new.append((k, v))
        return x @ self.head, torch.stack([a for a, _ in new]), torch.stack([a for _, a in new])

    def check(self, tokens, logits, plan, uniform, count):
        """Accepted paths and next tokens against the most likely ones."""
        b, n = tokens.shape
        target = torch.zeros((b, n, self.vocab), device=DEV)
        target.scatter_(2, logits.argmax(-1, keepdim=True), 1.0)
        path = torch.empty((b, n), dtype=torch.int32, device=DEV)
        got, nxt = (torch.empty(b, dtype=torch.int32, device=DEV) for _ in range(2))
        B.tree_verify(B.make_tree(n, count=count, plan=plan), tokens, target, None, uniform, path,
                      got, nxt)
        return path, got, nxt


def test_speculative_decoding_gives_the_sequential_tokens():
    batch, steps, n = 3, 30, 11
    rng = random.Random(7)
    g = torch.Generator().manual_seed(7)
    prompt = torch.randint(0, 53, (batch, 9), generator=g, dtype=torch.int32).to(DEV)

    def start():
        m = Toy(batch)
        tree = B.make_tree(9, ints([-9] * batch))
        logits, kn, vn = m.forward(prompt, tree)
        B.kv_append(m.p, m.s, tree, kn, vn, m.k, m.v, m.lay)
        return m, logits[:, -1].argmax(-1).int()

    # token by token
    m, tok = start()
    seq = [tok.tolist()]
    for t in range(steps):
        tree = B.make_tree(1, ints([t] * batch))
        logits, kn, vn = m.forward(tok[:, None], tree)
        B.kv_append(m.p, m.s, tree, kn, vn, m.k, m.v, m.lay)
        tok = logits[:, 0].argmax(-1).int()
        seq.append(tok.tolist())
    seq = np.array(seq).T  # [batch, steps + 1]

    # with drafts: now and then the right token, sometimes two of a kind
    s, tok = start()
    base = ints([0] * batch)
    have = [[int(x)] for x in tok]
    plan = torch.empty(B.tree_plan_bytes(batch, n), dtype=torch.uint8, device=DEV)
    calls, longest = 0, 0
    while min(len(h) for h in have) <= steps:
        parents = [random_parents(rng, n, 3) for _ in range(batch)]
        drafts = np.zeros((batch, n), np.int32)
        counts = []
        for b in range(batch):
            drafts[b, 0] = have[b][-1]
            done = len(have[b]) > steps
            counts.append(0 if done else rng.randint(1, n))
            for i in range(1, n):
                at = len(have[b]) - 1 + len(otree.line(parents[b], i)) - 1
                right = seq[b][at] if at <= steps else 0
                drafts[b, i] = right if rng.random() < 0.6 else rng.randrange(53)
        count, tokens = ints(counts), ints(drafts.tolist())
        B.tree_plan(ints(parents), count, plan)
        tree = B.make_tree(n, base, count, plan)
        logits, kn, vn = s.forward(tokens, tree)
        path, got, nxt = s.check(tokens, logits, plan,
                                 torch.rand((batch, n + 1), generator=g).to(DEV), count)
        B.kv_append(s.p, s.s, tree, kn, vn, s.k, s.v, s.lay, path, got)
        base = base + got
        for b in range(batch):
            if counts[b]:
                line = [x for x in path[b].tolist() if x >= 0]
                assert line[0] == 0 and len(line) == int(got[b])
                have[b] += [int(drafts[b, i]) for i in line[1:]] + [int(nxt[b])]
                longest = max(longest, len(line))
            else:
                assert int(got[b]) == 0 and int(nxt[b]) == -1
        calls += 1
    assert longest > 2 and calls < steps
    for b in range(batch):
        assert have[b][:steps + 1] == seq[b].tolist()
        # The first layer's rows depend on the tokens alone. Each side is a
        # library's sum of 256 products in fp32, whose order follows the number
        # of rows (off by at most 256 * 2^-24 of the sum of the magnitudes), and
        # rounded to bf16 (off by at most 2^-8 of it): twice both apart.
        rows = 9 + steps
        ids = torch.cat([prompt[b].long().cpu(), torch.from_numpy(seq[b][:steps])]).to(DEV)
        size = (m.emb[ids].abs().double() @ m.w[0].abs().double()).view(rows, -1, 64)
        exact = (m.emb[ids].double() @ m.w[0].double()).view(rows, -1, 64)
        band = 2.0 ** -8 * exact.abs() + (1 + 2.0 ** -8) * 256 * 2.0 ** -24 * size
        for x, at in ((m.k, 4), (s.k, 4), (m.v, 6), (s.v, 6)):
            err = (x[0, b, :, :rows].transpose(0, 1).double() - exact[:, at:at + 2]).abs()
            assert (err <= band[:, at:at + 2]).all()


def test_appended_rows_feed_a_decode_step():
    """A sparse decode step over a ring cache that kv_append filled equals the
    step over the same cache written by hand."""
    batch, hkv, d, lp, grid = 2, 4, 64, 11, (8, 8)
    p = B.make_params(lp, *grid, 24, 9, B.MODE_DIAGONAL, 2)
    s = B.make_shape(batch, hkv, hkv, d)
    ring = 2 + 24
    g = torch.Generator().manual_seed(5)
    x = torch.randn((batch, lp + 50, 2 * hkv, d), generator=g).bfloat16().to(DEV)
    q = torch.randn((50, batch, hkv, d), generator=g).bfloat16().to(DEV)
    results = []
    for own in (True, False):
        k, v = (torch.zeros((batch, hkv, lp + ring, d), dtype=torch.bfloat16, device=DEV)
                for _ in range(2))
        lay = B.kv_layout(k, ring_rows=ring)
        bufs = B.alloc_buffers(p, s, DEV)
        B.state_reset(p, s, bufs.state)
        outs = []
        for t in [None] + list(range(50)):
            part = slice(0, lp) if t is None else slice(lp + t, lp + t + 1)
            kn, vn = x[:, part, :hkv], x[:, part, hkv:]
            if own:
                tree = B.make_tree(kn.shape[1], ints([-lp if t is None else t] * batch))
                B.kv_append(p, s, tree, kn, vn, k, v, lay)
            else:
                row = slice(0, lp) if t is None else lp + (t if t < 2 else 2 + (t - 2) % 24)
                if t is None:
                    k[:, :, row], v[:, :, row] = kn.transpose(1, 2), vn.transpose(1, 2)
                else:
                    k[:, :, row], v[:, :, row] = kn[:, 0], vn[:, 0]
            if t is not None:
                B.decode_step(p, s, q[t], k, v, lay, ints([t] * batch), bufs.state, bufs.plan, 0.125,
                              bufs.out, bufs.logits, bufs.workspace)
                outs.append(bufs.out.clone())
        results.append(torch.stack(outs))
    assert torch.equal(results[0], results[1])


@pytest.mark.parametrize("given", [1, 5, 8, 9, 12])
def test_known_tokens_before_a_diagonal_run(given):
    """An image's first tokens in one dense chunk, then diagonal steps: with up to
    N_att - 1 of them every later step is what it is after single steps, and the
    chunk's outputs are the steps' (both fp32, the steps' weights in two bf16 terms:
    2^-15 apart); with more the next step is flagged."""
    batch, hkv, d, lp, grid, n_att = 2, 4, 64, 11, (8, 8), 9
    p = B.make_params(lp, *grid, 24, n_att, B.MODE_DIAGONAL, 2)
    dense = B.make_params(lp, *grid, 1, 1, B.MODE_DENSE)
    s = B.make_shape(batch, hkv, hkv, d)
    g = torch.Generator().manual_seed(6)
    x = torch.randn((batch, lp + 40, 2 * hkv, d), generator=g).bfloat16().to(DEV)
    q = torch.randn((40, batch, hkv, d), generator=g).bfloat16().to(DEV)
    results, flags = [], []
    for n in (0, given):
        k, v = (torch.zeros((batch, hkv, lp + 64, d), dtype=torch.bfloat16, device=DEV)
                for _ in range(2))
        lay = B.kv_layout(k)
        bufs = B.alloc_buffers(p, s, DEV)
        B.state_reset(p, s, bufs.state)
        append = lambda a, b: B.kv_append(  # noqa: E731
            p, s, B.make_tree(b - a, ints([a - lp] * batch)), x[:, a:b, :hkv], x[:, a:b, hkv:], k,
            v, lay)
        append(0, lp)
        out = torch.zeros((batch, 40, hkv, d), device=DEV)
        if n:
            size = B.tree_workspace_bytes(dense, s, n)
            ws = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None
            part = torch.empty((batch, n, hkv, d), device=DEV)
            B.tree_attention(dense, s, B.make_tree(n, ints([0] * batch)),
                             q[:n].transpose(0, 1).contiguous(), x[:, lp:lp + n, :hkv],
                             x[:, lp:lp + n, hkv:], k, v, lay, 0.125, part, ws)
            out[:, :n] = part
            append(lp, lp + n)
        behind = []
        for t in range(n, 40):
            append(lp + t, lp + t + 1)
            B.decode_step(p, s, q[t], k, v, lay, ints([t] * batch), bufs.state, bufs.plan, 0.125,
                          bufs.out, bufs.logits, bufs.workspace)
            out[:, t] = bufs.out
            behind.append(bool((B.state_views(p, s, bufs.state)[1] & B.FLAG_STATE_BEHIND).any()))
        results.append(out)
        flags.append(behind)
    assert not any(flags[0])
    if given < n_att:
        assert not any(flags[1])
        assert torch.equal(results[0][:, given:], results[1][:, given:])
        assert (results[0] - results[1]).abs().max() <= 2 ** -15 * x[..., hkv:, :].abs().max()
    else:
        assert flags[1][0]
