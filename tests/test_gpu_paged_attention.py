"""Attention over pages against fp64: modes, types, heads, lengths, pages, and
what must not reach an output."""

import itertools
import math

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.paged_util import Attend

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kv,d,group", itertools.product(("bf16", "fp8"), (64, 128), (1, 2, 4, 8)))
def test_types_and_heads(kv, d, group):
    for i, (mode, out) in enumerate((("dense", "fp32"), ("window", "bf16"), ("diagonal", "fp32"))):
        x = Attend(batch=3, heads=(2 * group, 2), d=d, kv=kv, mode=mode, out=out, grid=(9, 11),
                   n_att=30, sinks=4 * (i > 0), window=50, seed=10 * group + i)
        x.run()
        x.check()


@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 128, 1024])
@pytest.mark.parametrize("mode", ["dense", "window", "diagonal"])
def test_pages_of_any_size(page, mode):
    x = Attend(batch=3, heads=(4, 2), page=page, mode=mode, n_att=40, sinks=4, window=70,
               grid=(11, 13), prompts=[21, 0, 13], seed=page)
    x.run()
    x.check()


@pytest.mark.parametrize("prompt", [0, 1, 15, 16, 31, 32, 33, 130])
def test_lengths(prompt):
    """Every short position, and those around tiles' and pages' ends."""
    at = [0, 1, 2, 14, 15, 16, 17, 30, 31, 32, 33, 63, 64, 65, 98, -1]
    for kv in ("bf16", "fp8"):
        x = Attend(batch=len(at), heads=(2, 2), prompt=prompt, pos=at, kv=kv, seed=prompt)
        x.run()
        x.check()


@pytest.mark.parametrize("mode", ["dense", "window", "diagonal"])
def test_long_rows_are_split(mode):
    for kv, group, d in (("bf16", 1, 128), ("fp8", 4, 64), ("bf16", 8, 64)):
        x = Attend(batch=2, heads=(2 * group, 2), d=d, prompt=300, grid=(60, 61), page=32,
                   pos=[3659, 1500], mode=mode, n_att=1500, sinks=4, window=2500, kv=kv,
                   prompts=[300, 177], seed=group)
        assert B.paged_launch_info(x.p, x.s).max_splits > 1
        x.run()
        x.check()


def test_unused_slots_and_positions_past_the_grid():
    x = Attend(batch=4, pos=[-1, 98, 99, 1000], seed=5)
    x.run()
    x.check()
    assert (x.out[0] == 0).all()
    y = Attend(batch=4, pos=[-5, 98, 98, 98], seed=5)
    y.run()
    y.check()


def test_prompt_lengths_are_clamped():
    x = Attend(batch=3, prompts=[-4, 1000, 7], seed=6)
    x.run()
    x.check()


@pytest.mark.parametrize("mode", ["dense", "window", "diagonal"])
@pytest.mark.parametrize("holes", [0.3, 1.0])
def test_rows_without_a_page(mode, holes):
    """Left out; with none left the output is 0 and the logits -infinity."""
    for kv in ("bf16", "fp8"):
        x = Attend(batch=3, heads=(4, 2), page=8, mode=mode, n_att=40, sinks=4, window=70,
                   holes=holes, kv=kv, seed=3)
        x.run()
        x.check()
        if holes == 1.0:
            assert (x.out == 0).all()


def test_entries_outside_the_pool_name_no_page():
    x = Attend(batch=3, heads=(4, 2), page=8, holes=0.4, seed=4)
    t = x.pages.table
    bad = torch.tensor([-1, -2, x.k.shape[0], 1 << 30, -(1 << 31)], dtype=torch.int32, device="cuda")
    at = (t < 0).nonzero()
    for i, (b, e) in enumerate(at.tolist()):
        t[b, e] = bad[i % len(bad)]
    x.run()
    x.check()


def test_rows_past_the_tables_row_are_left_out():
    x = Attend(batch=2, heads=(2, 2), page=8, pos=[98, 60], width=9, seed=8)
    x.run()
    x.check()


@pytest.mark.parametrize("hidden", [NAN, INF, -INF, 3e38])
@pytest.mark.parametrize("mode", ["dense", "window", "diagonal"])
def test_what_is_hidden_stays_hidden(hidden, mode):
    for group in (1, 4):
        x = Attend(batch=3, heads=(2 * group, 2), mode=mode, n_att=30, sinks=2, window=60,
                   holes=0.2, hidden=hidden, seed=group)
        x.run()
        x.check()
    x = Attend(batch=3, heads=(4, 2), mode=mode, n_att=30, sinks=2, window=60, holes=0.2, kv="fp8",
               hidden=448.0 if hidden == 3e38 else NAN, seed=9)
    x.run()
    x.check()


@pytest.mark.parametrize("order", ["page", "head", "row"])
def test_strides(order):
    for kv in ("bf16", "fp8"):
        x = Attend(batch=3, heads=(4, 2), order=order, kv=kv, seed=2)
        x.run()
        x.check()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 5.0, 40.0])
def test_scales(scale):
    x = Attend(batch=2, heads=(4, 2), scale=scale, seed=2)
    x.run()
    x.check()


def test_fp8_without_scales():
    x = Attend(batch=2, heads=(4, 2), kv="fp8", scales=False, seed=2)
    x.run()
    x.check()


def test_large_and_small_scores():
    """Queries and keys of 2^40: scores far apart, one row takes all the weight;
    and equal scores: the mean."""
    x = Attend(batch=2, heads=(2, 2), seed=2)
    x.q.mul_(2.0 ** 40)
    x.run()
    x.check()
    x.q.zero_()
    x.run()
    x.check()


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("group", [1, 4])
def test_values_that_are_not_finite_show(value, group):
    """In an attended V row: that element of that KV head's outputs and no other."""
    for out in ("fp32", "bf16"):
        x = Attend(batch=2, heads=(2 * group, 2), pos=[60, 70], out=out, seed=3)
        want = x.run().clone()
        x.check()
        row = x.rows[0][1][33]
        x.v[x.table[0][row // x.page], 1, row % x.page, 5] = value
        x.run()
        hit = torch.zeros_like(x.out, dtype=torch.bool)
        hit[0, group:, 5] = True
        assert not x.out[hit].isfinite().any()
        assert torch.equal(x.out[~hit], want[~hit])


def test_keys_that_are_not_finite_show():
    x = Attend(batch=2, heads=(2, 2), pos=[60, 70], seed=3)
    want = x.run().clone()
    row = x.rows[1][0][3]
    x.k[x.table[1][row // x.page], 0, row % x.page, 5] = NAN
    x.run()
    assert x.out[1, 0].isnan().all()
    want[1, 0] = x.out[1, 0] = 0
    assert torch.equal(x.out, want)


def test_scores_of_minus_infinity():
    """One: no weight.  All: an output of 0."""
    x = Attend(batch=1, heads=(1, 1), pos=[40], seed=4)
    x.q.fill_(0)
    x.q[..., 0] = 1
    at = [(x.table[0][r // x.page], r % x.page) for r in x.rows[0][0]]
    for g, o in at[1:]:
        x.k[g, 0, o, 0] = -INF
    x.run()
    assert torch.equal(x.out[0, 0], x.v[at[0][0], 0, at[0][1]].float())
    x.k[at[0][0], 0, at[0][1], 0] = -INF
    x.run()
    assert (x.out == 0).all()


def test_pages_past_two_gib():
    """Offsets of more than 32 bits, in elements and bytes."""
    pages, page, d = 70000, 128, 128  # 4.6 GB of K in fp8, 2.3e9 elements x 2 heads
    k = torch.zeros((pages, 4, page, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros_like(k)
    x = Attend(batch=2, heads=(8, 4), d=d, page=page, grid=(20, 20), kv="fp8", seed=5)
    move = {}
    for b, line in enumerate(x.table):
        for i, g in enumerate(line):
            if g >= 0:
                move[g] = pages - 1 - 9 * len(move)
                x.pages.table[b, i] = move[g]
    for g, to in move.items():
        k.view(torch.uint8)[to] = x.k.view(torch.uint8)[g]
        v.view(torch.uint8)[to] = x.v.view(torch.uint8)[g]
    x.k, x.v, x.layout = k, v, B.page_layout(k, x.k_scale, x.v_scale)
    x.run()
    x.check()


def test_same_results_every_time():
    x = Attend(batch=3, heads=(8, 2), d=128, grid=(40, 40), seed=6)
    want = x.run().clone()
    for _ in range(5):
        x.ws.fill_(255) if x.ws is not None else None
        assert torch.equal(x.run(), want)


def test_graph_replays_follow_table_and_positions():
    x = Attend(batch=3, heads=(4, 2), grid=(30, 31), pos=[900, 3, 77], prompts=[21, 4, 9], seed=7)
    y = Attend(batch=3, heads=(4, 2), grid=(30, 31), pos=[5, 800, -1], prompts=[2, 21, 9], seed=8)
    want = [z.run().clone() for z in (x, y)]
    x.check()
    y.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.run()
    mine = [t.clone() for t in (x.k, x.v, x.q, x.pages.table, x.pages.prompt, x.pos_t)]
    other = (y.k, y.v, y.q, y.pages.table, y.pages.prompt, y.pos_t)
    for i in (0, 1, 1, 0, 1):
        for to, value in zip((x.k, x.v, x.q, x.pages.table, x.pages.prompt, x.pos_t),
                             other if i else mine):
            to.copy_(value)
        x.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x.out, want[i])


def test_two_calls_at_once_and_two_graphs_with_one_workspace():
    a = Attend(batch=1, heads=(4, 4), d=128, grid=(50, 50), pos=[2400], seed=1)
    b = Attend(batch=1, heads=(4, 4), d=128, grid=(50, 50), pos=[1700], kv="fp8", out="bf16", seed=2)
    assert a.ws is not None
    want = []
    for x in (a, b):
        x.run()
        x.check()
        want.append(x.out.clone())
    outs = [[torch.full_like(x.out, 7.0) for _ in range(20)] for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for i in range(20):
        for x, st, got in zip((a, b), streams, outs):
            x.out = got[i]
            x.run(stream=st)
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(y, w) for y in got)
    b.ws = a.ws
    graphs = []
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for x in (a, b):
            x.out.fill_(7.0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
        a.ws.fill_(255)


def test_dense_pages_in_order_are_the_linear_cache():
    """The same rows through decode_attention: both are within their bounds of fp64,
    so within the sum of them of each other."""
    x = Attend(batch=2, heads=(8, 2), d=128, page=16, grid=(20, 20), pos=[399, 250], prompt=16,
               hidden=0.0, seed=9)
    x.run()
    x.check()
    rows = 16 + 400
    lin = [torch.zeros((2, 2, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for b in range(2):
        for i, g in enumerate(x.table[b]):
            if g >= 0:
                n = min(16, rows - 16 * i)
                lin[0][b, :, 16 * i:16 * i + n] = x.k[g, :, :n]
                lin[1][b, :, 16 * i:16 * i + n] = x.v[g, :, :n]
    out = torch.zeros_like(x.out)
    n = B.workspace_bytes(x.p, x.s)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    B.decode_attention(x.p, x.s, x.q, lin[0], lin[1], B.kv_layout(lin[0]), x.pos_t, None,
                       1 / math.sqrt(128), out, workspace=ws)
    assert (x.out - out).abs().max() <= 2e-5 * out.abs().max()


def test_an_out_buffer_is_all_that_is_written():
    x = Attend(batch=2, heads=(4, 2), grid=(30, 30), seed=3)
    whole = torch.full((x.out.numel() + 512,), 7.0, device="cuda")
    x.out = whole[256:256 + x.out.numel()].view(x.out.shape)
    before = [t.clone() for t in (x.k.view(torch.int16), x.v.view(torch.int16), x.pages.table)]
    x.run()
    x.check()
    assert (whole[:256] == 7).all() and (whole[256 + x.out.numel():] == 7).all()
    after = (x.k.view(torch.int16), x.v.view(torch.int16), x.pages.table)
    assert all(torch.equal(p, q) for p, q in zip(before, after))


def test_no_requests_of_work():
    x = Attend(batch=2, pos=[-1, -1], seed=3)
    x.run()
    assert (x.out == 0).all()
    y = Attend(batch=1, prompt=0, grid=(1, 1), pos=[0], seed=3)
    y.run()
    y.check()
    assert torch.equal(y.out[0], y.v[y.table[0][0], :, 0].float())


def test_plan_rows_out_of_range_are_clamped():
    """As in the decode kernels: a corrupt plan reads valid rows."""
    x = Attend(batch=1, heads=(2, 2), mode="diagonal", n_att=10, window=20, pos=[50], page=8,
               hidden=0.5, holes=0.0, seed=3)
    count, _, places = B.plan_views(x.p, x.s, x.plan)
    places[0, 0], places[0, 1], count[1] = -7, 1 << 30, 1 << 20
    x.run()
    assert x.out.isfinite().all()
