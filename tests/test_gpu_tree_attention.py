"""``tree_plan`` and ``tree_attention`` against the fp64 oracle."""

import math
import random

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2609_19702_amd import binding as B
from tests.gpu_util import DEV, say
from tests.tree_util import Problem, random_parents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [1, 2, 31, 32, 33, 64, 200, 256])
def test_plan(nodes):
    rng = random.Random(nodes)
    rows = [random_parents(rng, nodes, b) for b in (1, 2, 4, 300)]
    rows.append(otree.chain(nodes))
    rows.append([-1] * nodes)
    counts = [nodes, max(1, nodes // 2), nodes, 0, nodes + 5, nodes]
    batch = len(rows)
    buf = torch.full((B.tree_plan_bytes(batch, nodes),), 0xAA, dtype=torch.uint8, device=DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    B.tree_plan(ints(rows), ints(counts), buf)
    flags, deepest, depth, parent, anc = (x.cpu().numpy()
                                          for x in B.tree_plan_views(batch, nodes, buf))
    assert not flags.any()
    for b in range(batch):
        n = min(counts[b], nodes)
        for i in range(n):
            up = otree.line(rows[b], i)
            assert depth[b, i] == len(up) - 1 and parent[b, i] == rows[b][i]
            bits = sum(int(w) % (1 << 32) << 32 * j for j, w in enumerate(anc[b, i]))
            assert bits == sum(1 << m for m in up)
        assert (parent[b, n:] == -1).all() and (depth[b, n:] == 0).all()
        assert deepest[b] == (max(depth[b, :n]) if n else 0)


def test_plan_flags_bad_parents():
    rows = torch.tensor([[-1, 0, 1, 2], [-1, 1, 0, 7], [0, 0, -5, 2]], dtype=torch.int32, device=DEV)
    buf = torch.empty(B.tree_plan_bytes(3, 4), dtype=torch.uint8, device=DEV)
    B.tree_plan(rows, None, buf)
    flags, deepest, depth, parent, anc = (x.cpu().tolist() for x in B.tree_plan_views(3, 4, buf))
    assert flags == [0, B.TREE_FLAG_BAD_PARENT, B.TREE_FLAG_BAD_PARENT]
    assert parent == [[-1, 0, 1, 2], [-1, -1, 0, -1], [-1, 0, -1, 2]]
    assert depth == [[0, 1, 2, 3], [0, 0, 1, 0], [0, 1, 0, 1]] and deepest == [3, 1, 1]


TREES = [
    # one token: a decode step
    dict(nodes=1),
    dict(nodes=1, tree=False, out="bf16", d=128),
    dict(nodes=7),
    dict(nodes=16, d=128, out="bf16", layout="heads"),
    dict(nodes=17, heads=(8, 4), d=128, layout="nodes"),
    dict(nodes=33, heads=(8, 2), out="bf16"),
    dict(nodes=61, heads=(8, 1), d=128, grid=(17, 19), branch=4),
    dict(nodes=64, heads=(16, 2), kv="fp8", grid=(17, 19), branch=2),
    dict(nodes=256, heads=(2, 2), grid=(20, 20), branch=2, out="bf16"),
    dict(nodes=130, heads=(4, 2), kv="fp8", d=128, out="bf16", branch=4),
    # no prompt, nothing cached, the whole image cached
    dict(nodes=5, prompt=0, bases=[0, 1]),
    dict(nodes=9, prompt=1, bases=[0, 99], kv="fp8"),
    dict(nodes=12, bases=[99, 500], out="bf16"),
    # ragged requests, unused slots
    dict(batch=6, nodes=19, counts=[19, 1, 0, 7, -3, 40], bases=[5, 0, 7, -22, 3, 80]),
    dict(batch=3, nodes=21, counts=[20, 5, 1], heads=(8, 1), kv="fp8", row_base=False),
    dict(batch=4, nodes=11, row_base=True, d=128),
    # windows: shorter than a tree is deep, one token, wider than the image
    dict(nodes=24, mode="window", n_att=1, branch=1),
    dict(nodes=24, mode="window", n_att=3, sinks=2, branch=1, bases=[0, 60]),
    dict(nodes=40, mode="window", n_att=12, sinks=4, bases=[1, 50], out="bf16"),
    dict(nodes=40, mode="window", n_att=12, sinks=4, branch=1, bases=[2, 57], kv="fp8"),
    dict(nodes=40, mode="window", n_att=400, sinks=4, heads=(8, 2)),
    dict(nodes=12, mode="window", n_att=40, sinks=4, ring=40, bases=[3, 87]),
    dict(nodes=12, mode="window", n_att=40, sinks=4, ring=55, bases=[41, 80], kv="fp8", d=128),
    dict(nodes=30, mode="window", n_att=33, sinks=0, ring=33, bases=[64, 70], heads=(8, 1),
         grid=(17, 19), out="bf16"),
]


@pytest.mark.parametrize("case", TREES, ids=range(len(TREES)))
def test_tree(case):
    pr = Problem(seed=3, **case)
    pr.run()
    say("  worst error over its bound", pr.check())


CHUNKS = [
    # prompts, whole or from the middle on, and into the image
    dict(nodes=21, bases=[-21, -21]),
    dict(nodes=40, bases=[-21, -4], d=128, out="bf16"),
    dict(nodes=150, prompt=100, bases=[-100, -37], heads=(4, 1), kv="fp8"),
    dict(nodes=300, bases=[0, 3], grid=(20, 20), out="bf16"),
    dict(nodes=300, bases=[-21, 30], grid=(20, 20), heads=(8, 2), counts=[300, 1]),
    dict(batch=3, nodes=129, bases=[-21, 0, -30], heads=(8, 1), d=128, out="bf16"),
    # windows and sinks: within a tile, over many, sinks among the new tokens
    dict(nodes=300, bases=[-21, 0], grid=(20, 20), mode="window", n_att=37, sinks=4),
    dict(nodes=300, bases=[2, 77], grid=(20, 20), mode="window", n_att=37, sinks=4, out="bf16"),
    dict(nodes=333, bases=[-20, 3], grid=(20, 20), mode="window", n_att=141, sinks=9, kv="fp8",
         d=128, heads=(4, 2)),
    dict(nodes=200, bases=[90, 150], grid=(20, 20), mode="window", n_att=50, sinks=4, ring=50),
    dict(nodes=200, bases=[0, 199], grid=(20, 20), mode="window", n_att=1, out="bf16"),
    dict(nodes=520, bases=[-21, 100], grid=(26, 26), mode="window", n_att=230, sinks=70,
         heads=(8, 1), counts=[517, 400]),
]


@pytest.mark.parametrize("case", CHUNKS, ids=range(len(CHUNKS)))
def test_chunk(case):
    pr = Problem(seed=5, tree=False, **case)
    pr.run()
    n = case["nodes"]
    nodes = None if n < 64 else sorted({0, 1, n // 3, n // 2 + 1, n - 2, n - 1, 62, 63, 64, 65,
                                        min(127, n - 1), min(128, n - 1), 36, 37, 38, 49, 50, 51})
    say("  worst error over its bound", pr.check(nodes))


def query_rows(case):
    hq, hkv = case.get("heads", (4, 4))
    return case["nodes"] * hq // hkv


MANY = [c for c in [dict(seed=3, **c) for c in TREES] +
        [dict(seed=5, tree=False, **c) for c in CHUNKS] if query_rows(c) > 64]


@pytest.mark.parametrize("case", MANY, ids=range(len(MANY)))
def test_many_row_tiles(case):
    """The same with so many heads that the rows go through LDS, 128 at a time."""
    hq, hkv = case.get("heads", (4, 4))
    tiles = -(-query_rows(case) // 32) * hkv * case.get("batch", 2)
    f = 512 // tiles + 1
    pr = Problem(**{**case, "heads": (hq * f, hkv * f)})
    assert B.tree_launch_info(pr.p, pr.s, pr.nodes).rows_per_tile == 128
    pr.run()
    n = case["nodes"]
    nodes = {0, 1, n // 3, n // 2 + 1, n - 2, n - 1, 31, 32, 63, 64, 65, 127, 128, 36, 37, 38}
    say("  worst error over its bound",
        pr.check(sorted(i for i in nodes if i < n), sorted({0, hkv * f // 2, hkv * f - 1})))


@pytest.mark.parametrize("d", [64, 128])
def test_equals_a_decode_step(d):
    """A single node attends what a decode step at its position attends."""
    pr = Problem(batch=3, nodes=1, d=d, heads=(8, 4), tree=False, bases=[0, 31, 97])
    out = pr.run().clone()
    for b, t in enumerate(pr.bases):  # the step finds its row in the cache
        pr.k[b, :, pr.prompt + t] = pr.kn[b, 0]
        pr.v[b, :, pr.prompt + t] = pr.vn[b, 0]
    bufs = B.alloc_buffers(pr.p, pr.s)
    B.decode_attention(pr.p, pr.s, pr.q.reshape(3, 8, d).contiguous(), pr.k, pr.v, pr.layout,
                       pr.base, None, pr.scale, bufs.out, None, bufs.workspace)
    # two fp32 results of the same sums, the decode step's weights in two bf16
    # terms (2^-17)
    assert (bufs.out - out[:, 0]).abs().max() <= (2 ** -15) * pr.v.abs().max()


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("order", ["padded", "tokens"])
def test_cache_strides(kv, order):
    """Rows that are not next to each other: padded ones (not 16-byte aligned in
    fp8), and a token-major cache."""
    pr = Problem(nodes=21, heads=(8, 2), kv=kv, d=128, seed=6)
    want = pr.run().clone()
    b, h, rows, d = pr.k.shape
    pr.out.fill_(7.0)
    for name in ("k", "v"):
        x = getattr(pr, name)
        if order == "padded":
            y = torch.zeros((b, h, rows, d + 8), dtype=x.dtype, device=DEV)[..., :d]
        else:
            y = torch.zeros((b, rows, h, d), dtype=x.dtype, device=DEV).transpose(1, 2)
        y.view(torch.uint8 if kv == "fp8" else torch.bfloat16).copy_(
            x.view(torch.uint8 if kv == "fp8" else torch.bfloat16))
        setattr(pr, name, y)
    pr.layout = B.kv_layout(pr.k, k_scale=pr.k_scale, v_scale=pr.v_scale)
    assert torch.equal(pr.run(), want)


def test_binding_refuses_wrong_tensors():
    pr = Problem(nodes=6, heads=(8, 4))
    ok = dict(q=pr.q, k_new=pr.kn, v_new=pr.vn, k=pr.k, v=pr.v, out=pr.out, workspace=pr.ws)

    def call(**kw):
        a = {**ok, **kw}
        B.tree_attention(pr.p, pr.s, kw.pop("tree", pr.tree), a["q"], a["k_new"], a["v_new"],
                         a["k"], a["v"], pr.layout, pr.scale, a["out"], a["workspace"])

    bad = [dict(q=pr.q.float()), dict(q=pr.q[:, :5]), dict(k_new=pr.kn[..., :32]),
           dict(q=pr.q.contiguous().transpose(2, 3)), dict(v_new=pr.vn.contiguous()),
           dict(k=pr.k[:, :, :10], v=pr.v[:, :, :10]), dict(k=pr.k.float()), dict(v=pr.v[:1]),
           dict(out=pr.out.half()), dict(out=pr.out[:, :5]), dict(out=pr.out.transpose(0, 1)),
           dict(q=pr.q.cpu()), dict(out=pr.out.cpu()), dict(k=pr.k.cpu(), v=pr.v.cpu()),
           dict(tree=B.make_tree(6, pr.base[:1], None, pr.tree_plan)),
           dict(tree=B.make_tree(6, None, None, pr.tree_plan)),
           dict(tree=B.make_tree(6, pr.base, None, pr.tree_plan[:64]))]
    for kw in bad:
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(ValueError):
        B.make_tree(6, pr.base.long())
    with pytest.raises(ValueError):
        B.tree_plan(pr.parent.long(), None, pr.tree_plan)
    with pytest.raises(B.DSAError):
        B.tree_plan(pr.parent, None, pr.tree_plan[:64])
    with pytest.raises(ValueError):  # linear caches that cannot hold the whole image
        B.kv_append(pr.p, pr.s, pr.tree, pr.kn, pr.vn, pr.k[:, :, :50], pr.v[:, :, :50], pr.layout)
    call()


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(scale):
    pr = Problem(nodes=20, heads=(8, 4), seed=9)
    pr.scale = scale
    pr.run()
    pr.check()


@pytest.mark.parametrize("ks,vs", [(0.0, 1.0), (-0.01, 0.01), (0.01, -0.01), (0.01, 0.0)])
def test_unusual_cache_scales(ks, vs):
    pr = Problem(nodes=20, heads=(8, 4), seed=9, kv="fp8")
    pr.k_scale[::2] = ks
    pr.v_scale[::2] = vs
    pr.run()
    pr.check()


def _poison(x, kind):
    x[...] = {"nan": math.nan, "inf": math.inf, "-inf": -math.inf}[kind]


@pytest.mark.parametrize("kind", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("tree,heads,out", [(True, (4, 4), "fp32"), (True, (8, 1), "bf16"),
                                            (False, (4, 4), "bf16"), (False, (8, 1), "fp32"),
                                            (False, (160, 160), "bf16"), (True, (512, 64), "fp32")])
def test_hidden_values_stay_hidden(kind, tree, heads, out):
    """What a node must not see may hold anything: rows past a request's count,
    cache rows that hold nothing yet, another branch's K and V, later tokens,
    and positions that its window has left."""
    n = 30 if tree else 90
    for mode in (dict(), dict(mode="window", n_att=20, sinks=4)):
        case = dict(batch=2, nodes=n, heads=heads, out=out, tree=tree, counts=[n, n - 5],
                    bases=[40, 23], seed=11, grid=(15, 15), **mode)
        want = Problem(**case)
        want.run()
        got = Problem(**case)
        bad = n // 2  # its descendants see it, nobody else
        for b in range(2):
            _poison(got.kn[b, n - 5 if b else n:], kind)
            _poison(got.vn[b, n - 5 if b else n:], kind)
            _poison(got.k[b, :, got.prompt + got.bases[b]:], kind)
            _poison(got.v[b, :, got.prompt + got.bases[b]:], kind)
            _poison(got.kn[b, bad], kind)
            _poison(got.vn[b, bad, :, 5:9], kind)
            if mode:  # seen at depth 0 only
                j = got.prompt + got.bases[b] - 15
                _poison(got.v[b, :, j, 3], kind)
        got.run()
        torch.cuda.synchronize()
        a, w = got.out.float().cpu(), want.out.float().cpu()
        for b in range(2):
            for i in range(n - 5 if b else n):
                up = otree.line(got.parents[b], i)
                p = got.bases[b] + len(up) - 1
                sees = bad in up and (not mode or p - (got.bases[b] + up.index(bad)) < 16)
                edge = bool(mode) and len(up) == 1
                if not sees and not edge:
                    assert torch.equal(a[b, i], w[b, i]), (b, i)
                elif edge:
                    clean = torch.arange(a.shape[-1]) != 3
                    assert torch.equal(a[b, i][:, clean], w[b, i][:, clean])
                    assert not a[b, i][:, 3].isfinite().any()
                else:
                    assert not a[b, i][:, 5:9].isfinite().any()


@pytest.mark.parametrize("batch", [2, 31, 64, 65])
@pytest.mark.parametrize("nodes", [5, 17, 91])
def test_ragged_batches(batch, nodes):
    """Every request gets its own output, whatever the order they are worked in:
    equal ones, unused ones, prompts and full images side by side."""
    rng = random.Random(batch)
    bases = [rng.choice([0, 17, 17, 99, -21, -5, -30]) for _ in range(batch)]
    counts = [rng.choice([0, 1, nodes, nodes]) for _ in range(batch)]
    pr = Problem(batch=batch, nodes=nodes, heads=(8, 1), tree=False, bases=bases, counts=counts,
                 seed=batch)
    pr.run()
    pr.check(nodes=[0, nodes - 1])


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("nodes,heads", [(7, (4, 4)), (40, (8, 2)), (40, (256, 32))])
def test_nonfinite_value_in_the_last_row(kv, nodes, heads):
    """The last row that a cache has, in a tile with no keys after it: seen by all
    nodes, as the last of the new rows is by one."""
    for counts in (None, [nodes - 2, nodes]):
        case = dict(batch=2, nodes=nodes, heads=heads, tree=False, kv=kv, bases=[99, 99],
                    counts=counts, seed=4)
        want = Problem(**case)
        want.run()
        got = Problem(**case)
        if kv == "bf16":
            got.v[:, :, -1, 9] = math.inf
        else:
            got.v.view(torch.uint8)[:, :, -1, 9] = 0x7F
        for b in range(2):
            got.vn[b, (counts or [nodes] * 2)[b] - 1, :, 4] = -math.inf
        got.run()
        torch.cuda.synchronize()
        a, w = got.out.cpu(), want.out.cpu()
        for b in range(2):
            n = (counts or [nodes] * 2)[b]
            clean = [c for c in range(64) if c not in (4, 9)]
            assert torch.equal(a[b, :n][..., clean], w[b, :n][..., clean])
            if kv == "bf16":
                assert (a[b, :n, :, 9] == math.inf).all()
            else:
                assert a[b, :n, :, 9].isnan().all()
            assert torch.equal(a[b, :n - 1, :, 4], w[b, :n - 1, :, 4])
            assert (a[b, n - 1, :, 4] == -math.inf).all()
            assert torch.equal(a[b, n:], w[b, n:])


@pytest.mark.parametrize("nodes,heads,d", [(6, (4, 4), 64), (13, (8, 1), 128), (30, (8, 4), 128),
                                           (50, (8, 2), 64), (50, (256, 32), 64),
                                           (30, (512, 64), 128)])
@pytest.mark.parametrize("ring", [0, 20])
def test_hidden_fp8_codes_stay_hidden(nodes, heads, d, ring):
    """NaN codes of cached positions that some nodes' windows have left: those get
    the output that a zero in its place gives them, the others NaN."""
    case = dict(batch=2, nodes=nodes, heads=heads, d=d, tree=False, kv="fp8", mode="window",
                n_att=20, sinks=4, ring=ring, bases=[40, 61], grid=(11, 11), seed=8)
    want, got = Problem(**case), Problem(**case)
    for b in range(2):
        for back in (1, 4, 9, 16):  # position base - back: node i sees it where i + back < 16
            row = got.row_of(got.bases[b] - back)
            got.v.view(torch.uint8)[b, :, row, back + 30] = 0xFF if back & 1 else 0x7F
            want.v.view(torch.uint8)[b, :, row, back + 30] = 0
    want.run()
    got.run()
    torch.cuda.synchronize()
    a, w = got.out.cpu(), want.out.cpu()
    for i in range(nodes):
        for c in range(d):
            if c - 30 in (1, 4, 9, 16) and i + c - 30 < 16:
                assert a[:, i, :, c].isnan().all(), (i, c)
            else:
                assert torch.equal(a[:, i, :, c], w[:, i, :, c]), (i, c)


@pytest.mark.parametrize("nodes,heads", [(5, (4, 4)), (40, (8, 2)), (40, (256, 32))])
def test_visible_nan_is_a_nan(nodes, heads):
    """Also beside hidden keys, and next to infinities of one sign."""
    pr = Problem(nodes=nodes, heads=heads, tree=False, seed=2)
    pr.vn[:, 2, :, 7] = math.nan
    pr.vn[:, 3, :, 7] = math.inf
    pr.vn[:, 1, :, 8] = -math.inf
    pr.vn[:, 2, :, 8] = math.inf
    out = pr.run().cpu()
    assert out[:, 2:, :, 7].isnan().all() and out[:, 2:, :, 8].isnan().all()
    assert out[:, :2, :, 7].isfinite().all() and (out[:, 1, :, 8] == -math.inf).all()
    assert out[:, :, :, [c for c in range(64) if c not in (7, 8)]].isfinite().all()


def test_visible_infinity_is_an_infinity():
    """An infinite V element of a key that is seen gives that infinity, also in
    a tile with hidden keys."""
    pr = Problem(nodes=9, heads=(4, 4), parents=[[-1, 0, 0, 1, 1, 2, 3, 5, 6]] * 2)
    pr.vn[:, 2, :, 7] = math.inf
    pr.run()
    out = pr.out.cpu()
    for i in range(9):
        sees = 2 in otree.line(pr.parents[0], i)
        assert (out[:, i, :, 7] == math.inf).all() if sees else out[:, i].isfinite().all()
        assert out[:, i, :, :7].isfinite().all() and out[:, i, :, 8:].isfinite().all()


def test_strides_of_one_node_and_far_offsets():
    """A cache of more than 2^31 elements: the last requests' rows."""
    rows, batch = 70000, 4
    pr = Problem(batch=2, nodes=6, heads=(1, 1), d=128, prompt=8, grid=(8, 8))
    big = torch.zeros((batch, 64, rows, 128), dtype=torch.bfloat16, device=DEV)
    assert big.numel() > 2 ** 31
    bigv = torch.zeros_like(big)
    far = big.view(-1, rows, 128)[-2:].unsqueeze(1), bigv.view(-1, rows, 128)[-2:].unsqueeze(1)
    far[0][:, :, :72] = pr.k
    far[1][:, :, :72] = pr.v
    want = pr.run().clone()
    base = torch.tensor([(batch * 64 - 2) * rows * 128, (batch * 64 - 1) * rows * 128],
                        dtype=torch.int64, device=DEV)
    lay = B.KVLayout(base.data_ptr(), 0, 0, 128, 0, None, None, B.KV_BF16)
    pr.out.fill_(0)
    B.tree_attention(pr.p, pr.s, pr.tree, pr.q, pr.kn, pr.vn, big, bigv, lay, pr.scale, pr.out,
                     pr.ws)
    assert torch.equal(pr.out, want)


@pytest.mark.parametrize("case", [dict(nodes=16, d=128, batch=1, grid=(24, 24)),
                                  dict(nodes=64, heads=(8, 1), grid=(24, 24), kv="fp8"),
                                  dict(nodes=300, tree=False, grid=(24, 24), bases=[-21, 5]),
                                  dict(nodes=300, tree=False, grid=(24, 24), bases=[-21, 5],
                                       heads=(64, 64), d=128, kv="fp8")],
                         ids=["small", "grouped", "chunk", "many"])
def test_runs_repeat_and_replay(case):
    """Calls repeat bit for bit: again, on another stream, and from a captured
    graph whose inputs and base positions change between replays."""
    pr = Problem(seed=21, **case)
    first = pr.run().clone()
    assert torch.equal(pr.run(), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pr.out.fill_(7.0)
    side.wait_stream(torch.cuda.current_stream())
    pr.run(stream=side)
    side.synchronize()
    assert torch.equal(pr.out, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pr.run()
    wanted = []
    for step in range(4):
        pr.base.copy_(torch.tensor([max(0, x - 3 * step) if x >= 0 else x for x in pr.bases],
                                   dtype=torch.int32))
        pr.q.copy_(torch.randn_like(pr.q.float()).bfloat16())
        pr.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = pr.out.clone()
        pr.out.fill_(7.0)
        pr.run()
        torch.cuda.synchronize()
        assert torch.equal(pr.out, got), step
        wanted.append(got)
    assert not torch.equal(wanted[0], wanted[1])


def test_writes_stay_inside_their_buffers():
    """Guard bytes around the plan, the output and the workspace stay."""
    pr = Problem(nodes=37, heads=(8, 2), d=128, grid=(24, 24), counts=[37, 21], batch=2)

    def guarded(nbytes):
        buf = torch.full((nbytes + 512,), 0x5A, dtype=torch.uint8, device=DEV)
        return buf, buf[256:256 + nbytes]

    full = []
    for name in ("tree_plan", "ws"):
        if getattr(pr, name) is not None:
            buf, view = guarded(getattr(pr, name).numel())
            full.append(buf)
            setattr(pr, name, view)
    buf, view = guarded(pr.out.numel() * 4)
    full.append(buf)
    pr.out = view.view(torch.float32).view(pr.out.shape)
    pr.out.fill_(7.0)
    pr.tree = B.make_tree(pr.nodes, pr.base, pr.count, pr.tree_plan)
    pr.run()
    pr.check()
    for buf in full:
        assert (buf[:256] == 0x5A).all() and (buf[-256:] == 0x5A).all()
