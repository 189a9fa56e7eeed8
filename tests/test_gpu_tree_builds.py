"""Every build of the streaming attention kernel against the fp64 oracle: four and
eight waves, keys in few and many splits, head sizes, cache and output types.  Each
case asserts the launch that it is there for."""

import pytest

from paper_2609_19702_amd import binding as B
from tests.gpu_util import say
from tests.tree_util import Problem

pytestmark = pytest.mark.gpu

TYPES = [(d, kv, out) for d in (64, 128) for kv in ("bf16", "fp8") for out in ("fp32", "bf16")]


def launched(pr):
    info = B.tree_launch_info(pr.p, pr.s, pr.nodes)
    tiles = info.workgroups // info.splits  # row tiles of all pairs
    return info, 8 if tiles <= 256 else 4   # waves of a streaming workgroup


WINDOW = dict(mode="window", n_att=20, sinks=4)
FOUR = {
    # a row tile per pair, ragged counts, and the same with hidden cached keys
    "one tile": dict(batch=3, nodes=30, heads=(100, 100), counts=[30, 7, 19], bases=[60, 3, 88]),
    "window": dict(batch=3, nodes=30, heads=(100, 100), counts=[30, 0, 30], bases=[60, 50, -21],
                   branch=1, **WINDOW),
    # two row tiles per pair, the second one cut
    "groups": dict(batch=5, nodes=13, heads=(240, 60), counts=[13, 8, 9, 1, 13]),
    # more than 64 rows, all tiles on the chip at once
    "chain": dict(batch=1, nodes=70, heads=(100, 100), tree=False, bases=[41]),
    "ring": dict(batch=1, nodes=70, heads=(100, 100), tree=False, bases=[29], ring=25, **WINDOW),
}


@pytest.mark.parametrize("d,kv,out", TYPES)
@pytest.mark.parametrize("case", list(FOUR))
def test_four_waves(case, d, kv, out):
    pr = Problem(d=d, kv=kv, out=out, seed=31, **FOUR[case])
    info, waves = launched(pr)
    assert info.rows_per_tile == 32 and info.splits == 1 and waves == 4
    pr.run()
    n = pr.nodes
    say("  worst error over its bound",
        pr.check(sorted({0, 1, 6, 7, 8, n // 2, n - 2, n - 1}), [0, pr.hkv // 2, pr.hkv - 1]))


SPLIT = {
    "few": (dict(nodes=9, heads=(4, 4), grid=(40, 40), bases=[900]), 2, 8),
    "groups": (dict(nodes=17, heads=(8, 2), grid=(40, 40), bases=[1500]), 2, 8),
    "many": (dict(nodes=5, heads=(2, 1), grid=(90, 90), bases=[8000]), 9, 64),
    "many rows": (dict(nodes=40, heads=(2, 2), grid=(90, 90), bases=[7900], tree=False), 9, 64),
    # the last splits have no keys
    "short": (dict(nodes=5, heads=(2, 1), grid=(90, 90), bases=[3000]), 9, 64),
    "window": (dict(nodes=30, heads=(4, 4), grid=(40, 40), bases=[1400], mode="window",
                    n_att=700, sinks=4, branch=1), 2, 8),
}


@pytest.mark.parametrize("d,kv,out", TYPES)
@pytest.mark.parametrize("case", list(SPLIT))
def test_split_keys(case, d, kv, out):
    kw, least, most = SPLIT[case]
    pr = Problem(batch=1, d=d, kv=kv, out=out, seed=32, **kw)
    info, waves = launched(pr)
    assert info.rows_per_tile == 32 and least <= info.splits <= most and waves == 8
    pr.run()
    say("  worst error over its bound", pr.check(sorted({0, pr.nodes // 2, pr.nodes - 1}), [0]))
