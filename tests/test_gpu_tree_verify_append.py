"""``tree_verify`` and ``kv_append`` against the oracle: decisions and bytes are
equal, not close."""

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


class Verify:
    def __init__(self, batch, nodes, vocab, branch=3, draft=True, counts=None, seed=0, noise=1.0,
                 chain=False):
        rng = random.Random(seed)
        g = torch.Generator().manual_seed(seed)
        self.parents = [otree.chain(nodes) if chain else random_parents(rng, nodes, branch)
                        for _ in range(batch)]
        z = 2 * torch.randn((batch, nodes, vocab), generator=g)
        self.target = torch.softmax(z, -1)
        z = z + noise * torch.randn((batch, nodes, vocab), generator=g)
        self.draft = torch.softmax(z, -1) if draft else None
        self.tokens = torch.zeros((batch, nodes), dtype=torch.int32)
        for b in range(batch):
            for i in range(nodes):
                c = max(self.parents[b][i], 0)
                if draft:
                    self.tokens[b, i] = int(torch.multinomial(self.draft[b, c], 1, generator=g))
                else:  # likely tokens, now and then one twice
                    self.tokens[b, i] = int(z[b, c].topk(min(vocab, 3)).indices[rng.randrange(
                        min(vocab, 3))])
        self.uniform = torch.rand((batch, nodes + 1), generator=g)
        self.counts, self.chain = counts, chain

    def run(self, stream=None):
        t = self.target.to(DEV)
        batch, nodes, vocab = t.shape
        count = None if self.counts is None else ints(self.counts)
        plan = None
        if not self.chain:
            plan = torch.empty(B.tree_plan_bytes(batch, nodes), dtype=torch.uint8, device=DEV)
            B.tree_plan(ints(self.parents), count, plan)
        path = torch.full((batch, nodes), 77, dtype=torch.int32, device=DEV)
        got, tok = (torch.full((batch,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
        B.tree_verify(B.make_tree(nodes, None, count, plan), self.tokens.to(DEV), t,
                      None if self.draft is None else self.draft.to(DEV), self.uniform.to(DEV),
                      path, got, tok, stream=stream)
        return path, got, tok

    def check(self):
        path, got, tok = (x.cpu().tolist() for x in self.run())
        batch, nodes, vocab = self.target.shape
        kept = []
        for b in range(batch):
            n = nodes if self.counts is None else min(max(self.counts[b], 0), nodes)
            line, nxt = otree.verify(self.parents[b], self.tokens[b].tolist(),
                                     self.target[b].numpy(),
                                     None if self.draft is None else self.draft[b].numpy(),
                                     self.uniform[b].tolist(), n)
            assert path[b] == line + [-1] * (nodes - len(line)), b
            assert got[b] == len(line) and tok[b] == nxt, (b, tok[b], nxt)
            kept.append(len(line))
        return kept


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("nodes,vocab,branch,chain", [
    (1, 1, 1, False), (1, 5, 1, True), (2, 2, 1, False), (8, 63, 2, False), (9, 64, 1, True),
    (24, 1000, 3, False), (64, 1023, 4, False), (65, 1025, 9, False), (256, 300, 5, False),
    (17, 16384, 3, False), (5, 70001, 2, False)])
def test_verify(nodes, vocab, branch, chain, draft):
    kept = Verify(6, nodes, vocab, branch, draft, seed=nodes, chain=chain).check()
    # the inputs reach past the root (a likely token alone is seldom taken)
    assert nodes < 8 or not draft or max(kept) > 1


def test_verify_very_large_vocabulary():
    """More than 1024 blocks of 1024 tokens: blocks of several rounds."""
    Verify(1, 2, (1 << 20) + 12345, 1, True, seed=4).check()
    Verify(1, 2, (1 << 21) + 1, 1, False, seed=5).check()


def test_verify_ragged():
    Verify(7, 20, 257, 3, True, counts=[20, 1, 0, 5, -1, 33, 2], seed=2).check()


@pytest.mark.parametrize("draft", [True, False])
def test_verify_same_distribution_and_far_ones(draft):
    """A draft equal to the target is always accepted; one that the target never
    gives never is, and leaves the target's own distribution."""
    v = Verify(5, 6, 100, 1, True, seed=3, chain=True, noise=0.0)
    assert v.check() == [6] * 5
    v = Verify(5, 12, 100, 4, draft, seed=3)
    v.target[:, :, 50:] = 0
    v.tokens[:] = 60
    if draft:
        v.draft[:, :, :50] = 0
    assert v.check() == [1] * 5


def test_verify_degenerate_rows():
    """Rows without mass, drafts that leave none, NaN and negative entries,
    tokens outside the vocabulary, random numbers of 0 and next to 1."""
    v = Verify(8, 7, 40, 3, True, seed=8)
    v.target[0] = 0
    v.draft[1] = 1  # leaves nothing of any token
    v.target[2, :, ::2] = float("nan")
    v.draft[3, :, ::3] = -1.0
    v.tokens[4] = torch.tensor([0, -1, 40, 1 << 30, -(1 << 31), 5, 6])
    v.uniform[5] = 0.0
    v.uniform[6] = float(np.nextafter(np.float32(1), np.float32(0)))
    v.target[7] = 0
    v.target[7, :, 11] = 1.0
    v.check()
    v.draft = None
    v.check()


def test_verify_large_random_number_takes_the_last_token_with_mass():
    v = Verify(2, 1, 3000, 1, False, seed=1)
    v.target[:, :, 1777:] = 0
    v.uniform[:] = float(np.nextafter(np.float32(1), np.float32(0)))
    v.check()


def test_verify_keeps_the_targets_distribution():
    """Over many random numbers the first token after the root is distributed
    as the target's row, whatever the draft: 40 000 requests, five standard
    deviations of each token's count."""
    batch, vocab = 40000, 6
    g = torch.Generator(device=DEV).manual_seed(1)
    target = torch.tensor([0.4, 0.05, 0.25, 0.1, 0.0, 0.2], device=DEV)
    draft = torch.tensor([0.1, 0.3, 0.1, 0.2, 0.2, 0.1], device=DEV)
    n = 3  # the root and two samples of the draft
    tokens = torch.multinomial(draft, batch * n, True, generator=g).view(batch, n).int()
    plan = torch.empty(B.tree_plan_bytes(batch, n), dtype=torch.uint8, device=DEV)
    B.tree_plan(ints([[-1, 0, 0]] * batch), None, plan)
    path = torch.empty((batch, n), dtype=torch.int32, device=DEV)
    got, tok = (torch.empty(batch, dtype=torch.int32, device=DEV) for _ in range(2))
    B.tree_verify(B.make_tree(n, plan=plan), tokens, target.expand(batch, n, vocab).contiguous(),
                  draft.expand(batch, n, vocab).contiguous(),
                  torch.rand((batch, n + 1), generator=g, device=DEV), path, got, tok)
    second = torch.where(got > 1, tokens.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], tok)
    share = torch.bincount(second.long(), minlength=vocab).double() / batch
    band = 5 * (target.double() * (1 - target.double()) / batch).sqrt()
    assert (share - target.double()).abs().le(band).all(), (share, target)
    assert ((got > 1).double().mean() > 0.5).item()


def test_verify_replays():
    v = Verify(4, 12, 777, 3, True, seed=12)
    batch, nodes, vocab = v.target.shape
    t, d, x = v.target.to(DEV), v.draft.to(DEV), v.tokens.to(DEV)
    u, parent = v.uniform.to(DEV), ints(v.parents)
    plan = torch.empty(B.tree_plan_bytes(batch, nodes), dtype=torch.uint8, device=DEV)
    tree = B.make_tree(nodes, plan=plan)
    path = torch.empty((batch, nodes), dtype=torch.int32, device=DEV)
    got, tok = (torch.empty(batch, dtype=torch.int32, device=DEV) for _ in range(2))

    def call():
        B.tree_plan(parent, None, plan)
        B.tree_verify(tree, x, t, d, u, path, got, tok)

    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(4):
        u.copy_(torch.rand(u.shape, generator=torch.Generator().manual_seed(step)))
        g.replay()
        torch.cuda.synchronize()
        a = path.tolist(), got.tolist(), tok.tolist()
        call()
        torch.cuda.synchronize()
        assert a == (path.tolist(), got.tolist(), tok.tolist())
        v.uniform = u.cpu()
        v.check()


# ---- append --------------------------------------------------------------------

class Append:
    def __init__(self, layers=None, batch=3, hkv=4, d=64, prompt=13, grid=(6, 7), nodes=9,
                 bases=None, mode="dense", n_att=1, sinks=0, ring=0, kv="bf16", path=True,
                 accepted=None, counts=None, window=1, scales=True, seed=0, order=None):
        rng = random.Random(seed)
        g = torch.Generator().manual_seed(seed)
        self.batch, self.hkv, self.nodes, self.layers = batch, hkv, nodes, layers
        self.prompt, self.sinks, self.ring, self.length = prompt, sinks, ring, grid[0] * grid[1]
        self.mode = {"dense": B.MODE_DENSE, "window": B.MODE_WINDOW,
                     "diagonal": B.MODE_DIAGONAL}[mode]
        self.p = B.make_params(prompt, grid[0], grid[1], window, n_att, self.mode, sinks)
        self.s = B.make_shape(batch, hkv, hkv, d)
        lead = (layers,) if layers else ()
        rows = prompt + (ring or self.length)
        shape = lead + (batch, hkv, rows, d)
        self.scales = None
        if kv == "fp8":
            self.k, self.v = (torch.randint(0, 127, shape, generator=g, dtype=torch.uint8).to(DEV)
                              for _ in range(2))
            if scales:
                self.scales = [torch.rand(lead + (batch * hkv,), generator=g).to(DEV) * 0.01 + 0.001
                               for _ in range(2)]
        else:
            self.k, self.v = (torch.randn(shape, generator=g).bfloat16().to(DEV) for _ in range(2))
        x = torch.randn(lead + (batch, nodes, 2 * hkv, d), generator=g).bfloat16().to(DEV)
        self.kn, self.vn = x[..., :hkv, :], x[..., hkv:, :]
        self.bases = bases or [rng.randrange(0, max(1, self.length - nodes)) for _ in range(batch)]
        self.path = None
        if path:
            self.path = []
            for b in range(batch):
                at = sorted(rng.sample(range(nodes), rng.randint(1, nodes)))
                self.path.append(at + [-1] * (nodes - len(at)))
        self.accepted = accepted
        if path and accepted is None:
            self.accepted = [sum(i >= 0 for i in r) for r in self.path]
        self.counts = counts
        self.row_base = None
        self.order = order or list(range(batch))
        if order:
            step = self.k.stride(-4)
            self.row_base = torch.tensor([o * step for o in order], dtype=torch.int64, device=DEV)

    def layout(self):
        one = self.k[0] if self.layers else self.k
        ks, vs = self.scales or (None, None)
        return B.kv_layout(one, row_base=self.row_base, ring_rows=self.ring, k_scale=ks, v_scale=vs)

    def run(self):
        tree = B.make_tree(self.nodes, ints(self.bases),
                           None if self.counts is None else ints(self.counts))
        B.kv_append(self.p, self.s, tree, self.kn, self.vn, self.k, self.v, self.layout(),
                    None if self.path is None else ints(self.path),
                    None if self.accepted is None else ints(self.accepted))

    def check(self):
        """The whole caches, byte for byte."""
        before = [x.cpu().clone() for x in (self.k, self.v)]
        self.run()
        torch.cuda.synchronize()
        lead = range(self.layers) if self.layers else [None]
        for which, (want, got, new) in enumerate(zip(before, (self.k, self.v),
                                                     (self.kn, self.vn))):
            for la in lead:
                w = want if la is None else want[la]
                x = (new if la is None else new[la]).cpu()
                for b in range(self.batch):
                    n = self.nodes if self.counts is None else min(max(self.counts[b], 0),
                                                                   self.nodes)
                    if self.bases[b] < -self.prompt:
                        continue
                    take = n if self.accepted is None else min(max(self.accepted[b], 0), n)
                    for e in range(take):
                        pos = min(self.bases[b], self.length) + e
                        m = e if self.path is None else self.path[b][e]
                        if pos >= self.length or not 0 <= m < n:
                            continue
                        row = self.prompt + pos
                        if self.ring and self.ring < self.length and pos >= self.sinks:
                            row = self.prompt + self.sinks + (pos - self.sinks) % (self.ring -
                                                                                   self.sinks)
                        for h in range(self.hkv):
                            y = x[b, m, h]
                            if want.dtype is torch.uint8:
                                y = y.float()
                                if self.scales:
                                    sc = self.scales[which].cpu()
                                    sc = (sc if la is None else sc[la])[b * self.hkv + h]
                                    y = y / sc
                                y = torch.from_numpy(otree.encode_e4m3(y.numpy()))
                            w[self.order[b], h, row] = y
            assert torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))


APPENDS = [
    dict(),
    dict(nodes=1, path=False),
    dict(layers=5, d=128, hkv=3),
    dict(layers=3, kv="fp8"),
    dict(kv="fp8", scales=False, d=128),
    dict(path=False, nodes=13, bases=[-13, -13, -13], kv="fp8"),
    dict(path=False, nodes=30, bases=[-13, -4, 0], layers=2),
    dict(path=False, nodes=9, bases=[38, 42, 60]),             # over the image's end
    dict(bases=[-14, 3, -20], counts=[9, 9, 9]),               # unused slots
    dict(counts=[4, 0, -2], path=False),
    dict(accepted=[0, 9, 20]),
    dict(accepted=[-1, 2, 3], path=False, counts=[9, 1, 9]),
    dict(order=[2, 0, 1], kv="fp8"),
    dict(mode="window", n_att=12, sinks=4, ring=12, nodes=9, bases=[2, 20, 33]),
    dict(mode="window", n_att=12, sinks=4, ring=12, nodes=40, bases=[0, 1, -13], path=False),
    dict(mode="window", n_att=12, sinks=0, ring=15, nodes=40, bases=[0, 1, -13], path=False,
         kv="fp8", layers=2),
    dict(mode="diagonal", n_att=5, window=9, sinks=2, ring=11, nodes=6, bases=[0, 30, 39]),
    dict(mode="dense", ring=42, nodes=6),
]


@pytest.mark.parametrize("case", APPENDS, ids=range(len(APPENDS)))
def test_append(case):
    Append(seed=4, **case).check()


def test_append_skips_path_entries_outside_the_nodes():
    a = Append(nodes=6)
    a.path = [[0, 9, 2, -1, 5, 6], [-7, 1, 2, 3, 4, 5], [0, 1, 1 << 30, 3, 4, 5]]
    a.accepted = [6, 6, 6]
    a.check()


def test_append_rounds_as_the_format_does():
    """Values at and between E4M3 values, beyond the largest, tiny, infinite
    and NaN."""
    a = Append(batch=1, hkv=1, nodes=8, path=False, kv="fp8", scales=False)
    v = otree._VALUES
    mid = np.concatenate([v, (v[1:] + v[:-1]) / 2, [448, 460, 464, 1e9, np.inf, 2.0 ** -11,
                                                    2.0 ** -10, 1.5 * 2.0 ** -10, 0.0]])
    x = torch.from_numpy(np.concatenate([mid, -mid])).float()
    n = a.kn.numel()
    x = x.repeat(n // len(x) + 1)[:n].view(1, 8, 1, 64).bfloat16()
    a.kn.copy_(x)
    a.vn.copy_(x.flip(1))
    a.check()
    a.kn[0, 3, 0, 5] = float("nan")
    a.run()
    row = a.prompt + a.bases[0] + 3
    assert int(a.k[0, 0, row, 5]) & 0x7F == 0x7F and int(a.v[0, 0, row, 5]) & 0x7F != 0x7F


def test_append_replays():
    a = Append(kv="fp8", layers=3)
    base, path, got = ints(a.bases), ints(a.path), ints(a.accepted)
    tree, lay = B.make_tree(a.nodes, base), a.layout()
    call = lambda: B.kv_append(a.p, a.s, tree, a.kn, a.vn, a.k, a.v, lay, path, got)
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for step in range(4):
        a.bases = [min(step * 5 + b, 30) for b in range(a.batch)]
        base.copy_(torch.tensor(a.bases, dtype=torch.int32))
        k0, v0 = a.k.clone(), a.v.clone()
        g.replay()
        torch.cuda.synchronize()
        k1, v1 = a.k.clone(), a.v.clone()
        a.k.copy_(k0)
        a.v.copy_(v0)
        a.check()
        assert torch.equal(a.k, k1) and torch.equal(a.v, v1)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_append_into_padded_and_token_major_caches(kv):
    """Any row strides, and nothing written between the rows."""
    for order in ("padded", "tokens"):
        a = Append(kv=kv, layers=2)
        la, b, h, rows, d = a.k.shape
        want = Append(kv=kv, layers=2)
        want.run()
        full = []
        for name in ("k", "v"):
            x = getattr(a, name)
            if order == "padded":
                f = torch.full((la, b, h, rows, d + 8), 3, dtype=x.dtype, device=DEV)
                y = f[..., :d]
                full.append(f[..., d:])
            else:
                y = torch.zeros((la, b, rows, h, d), dtype=x.dtype, device=DEV).transpose(2, 3)
            y.copy_(x)
            setattr(a, name, y)
        a.run()
        assert torch.equal(a.k, want.k) and torch.equal(a.v, want.v)
        for f in full:
            assert (f == 3).all()


def test_verify_writes_its_outputs_only():
    v = Verify(5, 9, 100, seed=6)
    batch, nodes, vocab = v.target.shape
    plan = torch.empty(B.tree_plan_bytes(batch, nodes), dtype=torch.uint8, device=DEV)
    B.tree_plan(ints(v.parents), None, plan)
    full = torch.full((batch * (nodes + 2) + 192,), -77, dtype=torch.int32, device=DEV)
    path = full[64:64 + batch * nodes].view(batch, nodes)
    got = full[64 + batch * nodes:64 + batch * (nodes + 1)]
    tok = full[64 + batch * (nodes + 1):64 + batch * (nodes + 2)]
    B.tree_verify(B.make_tree(nodes, plan=plan), v.tokens.to(DEV), v.target.to(DEV),
                  v.draft.to(DEV), v.uniform.to(DEV), path, got, tok)
    want = v.run()
    assert torch.equal(path, want[0]) and torch.equal(got, want[1]) and torch.equal(tok, want[2])
    assert (full[:64] == -77).all() and (full[-128:] == -77).all()


def test_verify_binding_refuses_wrong_tensors():
    v = Verify(2, 4, 30, seed=1)
    t, d, u = v.target.to(DEV), v.draft.to(DEV), v.uniform.to(DEV)
    x = v.tokens.to(DEV)
    path = torch.empty((2, 4), dtype=torch.int32, device=DEV)
    got, tok = (torch.empty(2, dtype=torch.int32, device=DEV) for _ in range(2))
    tree = B.make_tree(4)
    ok = [tree, x, t, d, u, path, got, tok]
    bad = [(0, B.make_tree(5)), (1, x.long()), (1, x[:, :3]), (2, t.half()), (2, t[0]),
           (2, t.transpose(0, 1)), (3, d[..., :29]), (3, d.double()), (4, u[:, :4]),
           (5, path[:, :3]), (6, got[:1]), (7, tok.float()), (2, t.cpu()), (5, path.cpu())]
    for i, wrong in bad:
        with pytest.raises(ValueError):
            B.tree_verify(*[wrong if j == i else y for j, y in enumerate(ok)])
    with pytest.raises(ValueError):
        B.tree_verify(B.make_tree(4, count=got[:1]), *ok[1:])
    B.tree_verify(*ok)
