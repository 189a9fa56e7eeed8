"""Numbers of ``tree_attention`` where roundings, infinities and unusual scales
show: few keys, rows and codes that are not finite, every kernel."""

import math
import random

import numpy as np
import pytest
import torch

from oracle import tree as otree
from paper_2609_19702_amd import binding as B
from tests.gpu_util import say
from tests.tree_util import Problem

pytestmark = pytest.mark.gpu


# One request's short tree, with a workgroup per pair and with keys in splits,
# and rows that go through LDS 128 at a time.
KERNELS = {"whole": dict(batch=2, nodes=9), "split": dict(batch=1, nodes=9, grid=(40, 40)),
           "tiles": dict(batch=2, nodes=70, heads=(172, 172), tree=False)}


def problem(kernel, **kw):
    pr = Problem(**{**KERNELS[kernel], **kw})
    info = B.tree_launch_info(pr.p, pr.s, pr.nodes)
    assert (info.rows_per_tile == 128) == (kernel == "tiles")
    assert (info.splits > 1) == (kernel == "split")
    return pr


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kernel", list(KERNELS))
def test_bf16_outputs_round_the_result_alone(kernel, d, kv):
    """Few keys, so that no average hides what a weight is off by.  An element may
    be off by half a step of its own size, 2^-8 of it, by what fp32 arithmetic is
    (``band``), and by the weights' part: two bf16 terms, each nearest, leave
    2^-8 * 2^-8 of a weight, and the second term's products add n roundings of
    2^-24 to the sum over n keys."""
    pr = problem(kernel, d=d, kv=kv, out="bf16", prompt=2, bases=[1, 3][:KERNELS[kernel]["batch"]],
                 seed=d)
    pr.run()
    torch.cuda.synchronize()
    out = pr.out.double().cpu().numpy()
    k, v = pr.caches64()
    q, kn, vn = (x.double().cpu().numpy() for x in (pr.q, pr.kn, pr.vn))
    worst = 0.0
    for b in range(pr.batch):
        for i in range(min(9, pr.nodes)):
            held, up = otree.keys_of(pr.parents[b], i, pr.bases[b], pr.prompt, 0, None)
            rows = [pr.row_of(j) for j in held]
            for h in sorted({0, 1, pr.hkv - 1}):
                kk = np.concatenate([k[b, h, rows], kn[b, up, h]])
                vv = np.concatenate([v[b, h, rows], vn[b, up, h]])
                ref, band = otree.attend(q[b, i, h], kk, vv, pr.scale)
                e = (band + 2.0 ** -16 + len(kk) * 2.0 ** -24) * np.abs(vv).max()
                err = np.abs(out[b, i, h] - ref) / (2.0 ** -8 * (np.abs(ref) + e) + e)
                worst = max(worst, err.max())
    say("  worst error over its bound", worst)
    assert worst <= 1.0


CHAINS = {"stream": dict(batch=2, nodes=70, heads=(40, 40), grid=(15, 15), bases=[40, 90]),
          "split": dict(batch=1, nodes=70, heads=(4, 4), grid=(40, 40), bases=[900]),
          "four waves": dict(batch=1, nodes=70, heads=(100, 100), grid=(15, 15), bases=[90]),
          "tiles": dict(batch=2, nodes=200, heads=(172, 172), grid=(20, 20), bases=[40, 90])}


def chain(kernel, **kw):
    pr = Problem(tree=False, prompt=200, **CHAINS[kernel], **kw)
    info = B.tree_launch_info(pr.p, pr.s, pr.nodes)
    assert (info.rows_per_tile == 128) == (kernel == "tiles")
    assert (info.splits > 1) == (kernel == "split")
    assert (info.workgroups > 256) == (kernel in ("four waves", "tiles"))
    return pr


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kernel", list(CHAINS))
def test_seen_infinities_are_infinities_in_any_tile(kernel, d, out, kv):
    """Infinities and NaN of V rows in tiles that hide nothing, and where the
    weights underflow: node 60's key outweighs all others by hundreds of powers of
    two for about half of the queries.  What an element sees of them is what it is,
    the other elements are as without."""
    clean, pr = chain(kernel, d=d, out=out, kv=kv, seed=7), chain(kernel, d=d, out=out, kv=kv, seed=7)
    for x in (clean, pr):
        x.kn[:, 60] *= 1000
    if kv == "bf16":
        pr.v[:, :, 40, 5] = math.inf
        pr.v[:, :, 41, 6] = -math.inf
        pr.v[:, :, 42, 7] = math.inf
        pr.v[:, :, 100, 7] = -math.inf
        pr.v[:, :, 150, 8] = math.nan
    else:
        pr.v.view(torch.uint8)[:, :, 150, 8] = 0x7F
        pr.vn[:, 2, :, 8] = math.inf
    pr.vn[:, 3, :, 9] = math.inf
    pr.vn[:, 4, :, 10] = -math.inf
    pr.vn[:, 61, :, 10] = math.inf
    want, got = clean.run().cpu(), pr.run().cpu()
    full = {8: math.nan} if kv == "fp8" else {5: math.inf, 6: -math.inf, 7: math.nan, 8: math.nan}
    for c, x in full.items():
        assert (got[..., c].isnan() if math.isnan(x) else got[..., c] == x).all(), c
    assert (got[:, 3:, :, 9] == math.inf).all()
    assert (got[:, 4:61, :, 10] == -math.inf).all() and got[:, 61:, :, 10].isnan().all()
    same = torch.ones_like(got, dtype=torch.bool)
    same[..., list(full)] = False
    same[:, 3:, :, 9] = False
    same[:, 4:, :, 10] = False
    assert torch.equal(got[same], want[same]) and want.isfinite().all()


SCALED = {"stream": dict(nodes=30, heads=(4, 4)), "groups": dict(nodes=40, heads=(8, 2)),
          "split": dict(batch=1, nodes=30, heads=(4, 4), grid=(40, 40)),
          "tiles": dict(nodes=90, heads=(172, 172))}


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kernel", list(SCALED))
def test_nan_cache_scale_is_a_nan(kernel, d, which):
    """Of an fp8 cache: in every node that attends a cached row of the pair, and in
    no other one."""
    case = dict(grid=(12, 12), bases=[100, 60][:SCALED[kernel].get("batch", 2)], d=d, kv="fp8",
                tree=False, mode="dense", seed=d)
    case.update(SCALED[kernel])
    for window in (None, 7):
        if window:  # nodes from the seventh on attend new rows alone
            case.update(mode="window", n_att=7, prompt=0)
        clean, pr = Problem(**case), Problem(**case)
        pairs = torch.arange(pr.batch * pr.hkv, device=pr.k.device)
        getattr(pr, which)[pairs % 2 == 1] = math.nan
        want, got = clean.run().cpu(), pr.run().cpu()
        g = pr.hq // pr.hkv
        for b in range(pr.batch):
            for h in range(pr.hkv):
                bad = (b * pr.hkv + h) % 2 == 1
                n = min(pr.nodes, window - 1 if window else pr.nodes) if bad else 0
                assert got[b, :n, h * g:h * g + g].isnan().all(), (b, h)
                assert torch.equal(got[b, n:, h * g:h * g + g], want[b, n:, h * g:h * g + g]), (b, h)
        assert want.isfinite().all()


def test_layouts_with_too_few_scales_are_refused():
    """Before any kernel reads them: one layer's scales for an append of three layers,
    one request's for two, row bases likewise; scales of another type or order."""
    pr = Problem(nodes=6, kv="fp8")
    layers = 3
    k, v = (x.unsqueeze(0).repeat(layers, 1, 1, 1, 1) for x in (pr.k.view(torch.uint8),
                                                               pr.v.view(torch.uint8)))
    kn, vn = (x.unsqueeze(0).repeat(layers, 1, 1, 1, 1) for x in (pr.kn, pr.vn))
    scales = pr.k_scale.repeat(layers, 1)
    n = pr.k_scale.numel()

    def append(**kw):
        B.kv_append(pr.p, pr.s, pr.tree, kn, vn, k, v, B.kv_layout(k[0], **kw))

    for ks, vs in ((scales[0], scales[0]), (scales, scales[0]), (scales[1], None),
                   (scales[:2], scales)):
        with pytest.raises(ValueError):
            append(k_scale=ks, v_scale=vs)
    before = k.clone()
    append(k_scale=scales, v_scale=scales)
    assert not torch.equal(k, before)

    def attend(**kw):
        B.tree_attention(pr.p, pr.s, pr.tree, pr.q, pr.kn, pr.vn, pr.k, pr.v,
                         B.kv_layout(pr.k, **kw), pr.scale, pr.out, pr.ws)

    base = torch.zeros(1, dtype=torch.int64, device=pr.k.device)
    for kw in (dict(k_scale=pr.k_scale[:n - 1]), dict(v_scale=pr.v_scale[:1]),
               dict(row_base=base)):
        with pytest.raises(ValueError):
            attend(**kw)
    bufs = B.alloc_buffers(pr.p, pr.s)
    with pytest.raises(ValueError):
        B.decode_attention(pr.p, pr.s, pr.q[:, 0].contiguous(), pr.k, pr.v,
                           B.kv_layout(pr.k, k_scale=pr.k_scale[:1]), pr.base, None, pr.scale,
                           bufs.out, None, bufs.workspace)
    for kw in (dict(k_scale=pr.k_scale.half()), dict(v_scale=scales.t()),
               dict(k_scale=pr.k_scale.cpu()), dict(row_base=base.int())):
        with pytest.raises(ValueError):
            B.kv_layout(pr.k, **kw)
    attend(k_scale=pr.k_scale, v_scale=pr.v_scale)


ANYWHERE = [
    dict(batch=3, nodes=40, heads=(8, 2), bases=[40, 3, 95], counts=[40, 33, 1]),
    dict(batch=1, nodes=31, heads=(4, 4), bases=[700], grid=(40, 40), branch=1),
    dict(batch=2, nodes=61, heads=(256, 64), bases=[70, 12], branch=2),
    dict(batch=2, nodes=150, heads=(4, 1), bases=[-21, 60], grid=(15, 15), tree=False),
    dict(batch=2, nodes=150, heads=(172, 172), bases=[-13, 60], grid=(15, 15), tree=False),
]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("view", ["dense", "window", "ring"])
@pytest.mark.parametrize("case", range(len(ANYWHERE)))
def test_what_is_seen_of_rows_that_are_not_finite(case, view, kv):
    """Infinities and NaN in V rows anywhere, cached and new: an element is what its
    node sees of them, or as without them."""
    more = {"dense": {}, "window": dict(mode="window", n_att=25, sinks=4),
            "ring": dict(mode="window", n_att=25, sinks=4, ring=29)}[view]
    for d, out in ((64, "bf16"), (128, "fp32")):
        kw = dict(ANYWHERE[case], **more, kv=kv, d=d, out=out, seed=40 + case)
        clean, pr = Problem(**kw), Problem(**kw)
        rng = random.Random(case)
        kinds = {"inf": (1, 0), "-inf": (0, 1), "nan": (1, 1)}
        marks = []  # (request, position or None, node or None, column, what it gives)
        window = pr.window
        for b in range(pr.batch):
            base = pr.bases[b]
            for _ in range(8):
                lo = -pr.prompt if not pr.ring else max(-pr.prompt, base - 20)
                j, c = rng.randrange(lo, base) if base > lo else None, rng.randrange(d)
                if j is not None:
                    kind = "nan" if kv == "fp8" else rng.choice(list(kinds))
                    if kv == "fp8":
                        pr.v.view(torch.uint8)[b, :, pr.row_of(j), c] = 0x7F
                    else:
                        pr.v[b, :, pr.row_of(j), c] = float(kind)
                    marks = [m for m in marks if m[:2] + m[3:4] != (b, j, c)]
                    marks.append((b, j, None, c, kinds[kind]))
            for _ in range(8):
                m, c, kind = rng.randrange(pr.nodes), rng.randrange(d), rng.choice(list(kinds))
                pr.vn[b, m, :, c] = float(kind)
                marks = [x for x in marks if (x[0], x[2], x[3]) != (b, m, c)]
                marks.append((b, None, m, c, kinds[kind]))
        want, got = clean.run().float().cpu(), pr.run().float().cpu()
        for b in range(pr.batch):
            n = pr.nodes if pr.counts is None else pr.counts[b]
            for i in range(n):
                held, up = otree.keys_of(pr.parents[b], i, pr.bases[b], pr.prompt, pr.sinks, window)
                held, up = set(held), set(up)
                see = {}
                for _, j, m, c, what in (x for x in marks if x[0] == b):
                    if (m in up) if j is None else (j in held):
                        a = see.get(c, (0, 0))
                        see[c] = (a[0] | what[0], a[1] | what[1])
                w = want[b, i].clone()
                for c, (plus, minus) in see.items():
                    w[:, c] = math.nan if plus and minus else math.inf if plus else -math.inf
                assert torch.equal(got[b, i].nan_to_num(7e30), w.nan_to_num(7e30)), (b, i)
                assert torch.equal(got[b, i].isnan(), w.isnan()), (b, i)


@pytest.mark.parametrize("kernel", ["whole", "split", "tiles"])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
def test_infinite_keys(kernel, out):
    """A score of -inf takes its key out, one of +inf makes the row NaN, as the
    softmax does."""
    kw = dict(tree=False, out=out, prompt=40, bases=[30, 7][:KERNELS[kernel]["batch"]], seed=5)
    pr = problem(kernel, **kw)
    pr.k[:, :, 5, 0] = math.inf  # a score of the query's first element's sign
    sign = (pr.q[..., 0] > 0).cpu()
    got = pr.run().cpu()
    k, v = pr.caches64()
    q, kn, vn = (x.double().cpu().numpy() for x in (pr.q, pr.kn, pr.vn))
    for b in range(pr.batch):
        for i in sorted({0, 3, pr.nodes - 1}):
            held, up = otree.keys_of(pr.parents[b], i, pr.bases[b], pr.prompt, 0, None)
            rows = [r for r in (pr.row_of(j) for j in held) if r != 5]
            for h in sorted({0, 1, pr.hkv - 1}):
                x = got[b, i, h]
                if sign[b, i, h]:
                    assert x.isnan().all(), (b, i, h)
                    continue
                kk = np.concatenate([k[b, h, rows], kn[b, up, h]])
                vv = np.concatenate([v[b, h, rows], vn[b, up, h]])
                ref, band = otree.attend(q[b, i, h], kk, vv, pr.scale)
                e = (band + 2.0 ** -16 + len(kk) * 2.0 ** -24) * np.abs(vv).max()
                if out == "bf16":
                    e = 2.0 ** -8 * (np.abs(ref) + e) + e
                assert (np.abs(x.double().numpy() - ref) <= e).all(), (b, i, h)


@pytest.mark.parametrize("nodes,heads", [(9, (4, 4)), (40, (8, 2)), (90, (172, 172))])
def test_fp8_caches_without_scales(nodes, heads):
    """Scales of 1, exactly."""
    kw = dict(nodes=nodes, heads=heads, kv="fp8", grid=(15, 15), bases=[100, 60], seed=3)
    a, b = Problem(**kw), Problem(**kw)
    a.k_scale.fill_(1.0)
    a.v_scale.fill_(1.0)
    b.layout = B.kv_layout(b.k)
    assert torch.equal(a.run(), b.run())
