"""Tree calls at the same time on two streams, and two captured graphs on one."""

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.tree_util import Problem

pytestmark = pytest.mark.gpu

SPLIT = dict(batch=1, nodes=16, heads=(8, 8), d=128, grid=(40, 40))


def test_two_calls_at_once():
    """With workspaces of their own."""
    a, b = Problem(seed=1, **SPLIT), Problem(seed=2, kv="fp8", out="bf16", **SPLIT)
    assert B.tree_launch_info(a.p, a.s, a.nodes).splits > 1
    want = [x.run().clone() for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for x, st in zip((a, b), streams):
            x.run(stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


def test_two_graphs_share_a_workspace():
    """Captured one after the other, replayed in any order on one stream."""
    a, b = Problem(seed=3, **SPLIT), Problem(seed=4, **SPLIT)
    b.ws = a.ws
    want = [x.run().clone() for x in (a, b)]
    graphs = []
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        a.out.fill_(7.0)
        b.out.fill_(7.0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
        a.ws.fill_(255)


def test_each_of_two_calls_at_once_writes_its_results():
    """An output of its own, filled before, for every call on either stream; the
    expected ones are checked against fp64."""
    a, b = Problem(seed=1, bases=[900], **SPLIT), Problem(seed=2, kv="fp8", out="bf16", bases=[1200],
                                                         **SPLIT)
    want = []
    for x in (a, b):
        x.run()
        x.check(nodes=[0, 7, 15], kv_heads=[0, 7])
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
