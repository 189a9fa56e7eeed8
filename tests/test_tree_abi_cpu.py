"""Refusals and host logic of the calls that take several tokens per request;
no device work is launched here (every pointer is a made-up number, and every
call is refused before it is used)."""

import ctypes as C
import math

import pytest
import torch

from paper_2609_19702_amd import binding as B

PTR = 0x10000


def params(**kw):
    a = dict(prompt_len=20, grid_h=64, grid_w=64, window=1, n_att=1, mode=B.MODE_DENSE, sinks=0)
    a.update(kw)
    return B.make_params(**a)


def shape(batch=2, hq=8, hkv=4, d=64):
    return B.make_shape(batch, hq, hkv, d)


def tree(nodes=5, base=PTR, count=None, plan=None):
    return B.TreeRequest(nodes, base, count, plan)


ROWS = B.NodeRows(4096, 512, 64, 65536)


def layout(**kw):
    a = dict(d_row_base=None, stride_batch=61440, stride_head=7680, stride_row=64, ring_rows=0,
             d_k_scale=None, d_v_scale=None, dtype=B.KV_BF16)
    a.update(kw)
    return B.KVLayout(*[a[f[0]] for f in B.KVLayout._fields_])


def attention(p=None, s=None, t=None, q=PTR, qr=ROWS, kn=PTR, vn=PTR, nr=ROWS, k=PTR, v=PTR,
              kv=None, scale=0.1, out=PTR, out_type=0, ws=PTR, ws_bytes=1 << 40):
    p, s, t = p or params(), s or shape(), t if t is not None else tree()
    kv = kv or layout()
    ref = lambda x: None if x is False else C.byref(x)
    return B.lib().dsa_tree_attention(ref(p), ref(s), ref(t), q, ref(qr), kn, vn, ref(nr), k, v,
                                      ref(kv), scale, out, out_type, ws, ws_bytes, None)


INVALID = [
    dict(t=False), dict(t=tree(0)), dict(t=tree(-1)), dict(t=tree((1 << 20) + 1)),
    dict(t=tree(257, plan=PTR)), dict(t=tree(5, plan=PTR + 4)), dict(t=tree(base=None)),
    dict(q=None), dict(kn=None), dict(vn=None), dict(k=None), dict(v=None), dict(out=None),
    dict(qr=False), dict(nr=False), dict(q=PTR + 8), dict(kn=PTR + 2), dict(vn=PTR + 4),
    dict(k=PTR + 8), dict(v=PTR + 8), dict(out=PTR + 4),
    dict(qr=B.NodeRows(-8, 512, 64, 0)), dict(qr=B.NodeRows(8, 516, 64, 0)),
    dict(nr=B.NodeRows(8, 512, 63, 0)),
    dict(scale=math.inf), dict(scale=math.nan), dict(out_type=2), dict(out_type=-1),
    dict(kv=layout(dtype=2)), dict(kv=layout(stride_row=60)), dict(kv=layout(stride_row=68)),
    dict(kv=layout(d_k_scale=PTR)), dict(kv=layout(ring_rows=-1)), dict(kv=layout(ring_rows=50)),
    dict(p=params(mode=B.MODE_WINDOW, n_att=40), kv=layout(ring_rows=39)),
    dict(p=params(grid_h=0)), dict(p=params(mode=B.MODE_WINDOW, n_att=4, sinks=4)),
    dict(s=shape(hq=6)), dict(s=shape(batch=0)), dict(ws=PTR + 4),
    dict(s=shape(batch=4096), t=tree(1 << 19)),
]


@pytest.mark.parametrize("bad", INVALID, ids=range(len(INVALID)))
def test_attention_refuses(bad):
    if "ws" in bad:  # a launch that needs a workspace
        assert B.tree_workspace_bytes(params(), shape(1), 5) > 0
        bad = dict(bad, s=shape(1))
    assert attention(**bad) == B.ERR_INVALID_ARG


def test_attention_refuses_what_is_not_built():
    assert attention(p=params(mode=B.MODE_DIAGONAL, window=50, n_att=9)) == B.ERR_UNSUPPORTED
    assert attention(s=shape(d=96)) == B.ERR_UNSUPPORTED
    assert attention(s=shape(hq=12, hkv=4)) == B.ERR_UNSUPPORTED


def test_attention_refuses_a_short_workspace():
    p, s = params(), shape(1)
    need = B.tree_workspace_bytes(p, s, 5)
    assert need > 0
    assert attention(s=s, ws_bytes=need - 1) == B.ERR_WORKSPACE
    assert attention(s=s, ws=None) == B.ERR_WORKSPACE


def test_launch_info():
    for batch in (1, 2, 16, 64, 4096):
        for hq, hkv in ((8, 8), (8, 1), (20, 20)):
            for nodes in (1, 5, 16, 64, 256, 5000):
                if batch * hkv * nodes * hq // hkv > 1 << 24:
                    continue
                p, s = params(grid_h=64, grid_w=64), shape(batch, hq, hkv, 128)
                i = B.tree_launch_info(p, s, nodes)
                rows = nodes * (hq // hkv)
                assert (i.row_tiles - 1) * i.rows_per_tile < rows <= i.row_tiles * i.rows_per_tile
                assert i.workgroups == batch * hkv * i.row_tiles * i.splits
                assert (i.splits > 1) == (i.workspace_bytes > 0)
                assert i.workspace_bytes == B.tree_workspace_bytes(p, s, nodes)
                most = i.workgroups * i.rows_per_tile * (128 + 4) * 4
                assert i.workspace_bytes in (0, most)
    assert B.tree_workspace_bytes(params(mode=B.MODE_DIAGONAL, window=9, n_att=3), shape(), 4) == 0
    with pytest.raises(B.DSAError):
        B.tree_launch_info(params(), shape(), 0)


def test_plan_layout():
    for batch, nodes in ((1, 1), (3, 31), (2, 32), (5, 33), (64, 256)):
        L = B.tree_plan_layout(batch, nodes)
        assert L.words == (nodes + 31) // 32
        ends = [(L.flags_offset, 4 * batch), (L.max_depth_offset, 4 * batch),
                (L.depth_offset, 4 * batch * nodes), (L.parent_offset, 4 * batch * nodes),
                (L.ancestors_offset, 4 * batch * nodes * L.words), (L.bytes, 0)]
        for (a, n), (b, _) in zip(ends, ends[1:]):
            assert a % 256 == 0 and a + n <= b
        assert L.bytes == B.tree_plan_bytes(batch, nodes)
    for bad in ((0, 1), (1, 0), (1, 257), (1 << 30, 4)):
        assert B.tree_plan_bytes(*bad) == 0
        with pytest.raises(B.DSAError):
            B.tree_plan_layout(*bad)


def test_plan_refuses():
    f = B.lib().dsa_tree_plan
    need = B.tree_plan_bytes(2, 9)
    assert f(2, 9, None, None, PTR, need, None) == B.ERR_INVALID_ARG
    assert f(2, 9, PTR, None, None, need, None) == B.ERR_INVALID_ARG
    assert f(2, 257, PTR, None, PTR, 1 << 30, None) == B.ERR_INVALID_ARG
    assert f(2, 9, PTR, None, PTR + 8, need, None) == B.ERR_INVALID_ARG
    assert f(0, 9, PTR, None, PTR, need, None) == B.ERR_INVALID_ARG
    assert f(2, 9, PTR, None, PTR, need - 1, None) == B.ERR_WORKSPACE


def test_verify_refuses():
    def call(batch=2, vocab=100, t=None, ptrs=(PTR,) * 7):
        x, target, uniform, path, got, tok = ptrs[:6]
        t = tree(base=None) if t is None else t
        return B.lib().dsa_tree_verify(batch, vocab, C.byref(t) if t else None, x, target, None,
                                       uniform, path, got, tok, None)

    for bad in (dict(batch=0), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(t=False),
                dict(t=tree(257)), dict(t=tree(0))):
        assert call(**bad) == B.ERR_INVALID_ARG
    for i in range(6):
        assert call(ptrs=tuple(None if j == i else PTR for j in range(6))) == B.ERR_INVALID_ARG


def test_append_refuses():
    def call(p=None, s=None, t=None, kn=PTR, vn=PTR, nr=ROWS, layers=1, k=PTR, v=PTR, kv=None,
             sl=0):
        t = tree() if t is None else t
        ref = lambda x: None if x is False else C.byref(x)
        return B.lib().dsa_kv_append(C.byref(p or params()), C.byref(s or shape()), ref(t), kn, vn,
                                     ref(nr), None, None, layers, k, v, ref(kv or layout()), sl,
                                     None)

    for bad in (dict(t=False), dict(t=tree(0)), dict(t=tree(base=None)), dict(kn=None),
                dict(vn=None), dict(k=None), dict(v=None), dict(nr=False), dict(layers=0),
                dict(layers=-1), dict(sl=-8), dict(sl=12), dict(kn=PTR + 8), dict(k=PTR + 4),
                dict(nr=B.NodeRows(8, 8, 8, -8)), dict(nr=B.NodeRows(8, 8, 4, 8)),
                dict(kv=layout(ring_rows=50)), dict(kv=layout(dtype=7)), dict(s=shape(batch=0)),
                dict(t=tree(1 << 20), layers=1 << 30),
                dict(s=shape(1, 256, 256), t=tree(1 << 20))):
        assert call(**bad) == B.ERR_INVALID_ARG, bad
    assert call(s=shape(d=32)) == B.ERR_UNSUPPORTED


def test_binding_refuses_what_is_not_on_the_gpu():
    z = lambda *n, dtype=torch.int32: torch.zeros(n, dtype=dtype)
    with pytest.raises(ValueError):
        B.make_tree(4, z(2))
    with pytest.raises(ValueError):
        B.make_tree(4, None, z(2))
    with pytest.raises(ValueError):
        B.tree_plan(z(2, 4), None, z(4096, dtype=torch.uint8))
    t = B.make_tree(4, PTR)
    bf = torch.bfloat16
    k = z(2, 4, 120, 64, dtype=bf)
    with pytest.raises(ValueError):
        B.tree_attention(params(), shape(), t, z(2, 4, 8, 64, dtype=bf), z(2, 4, 4, 64, dtype=bf),
                         z(2, 4, 4, 64, dtype=bf), k, k, B.kv_layout(k), 0.1,
                         z(2, 4, 8, 64, dtype=bf))
    with pytest.raises(ValueError):
        B.tree_verify(t, z(2, 4), z(2, 4, 9, dtype=torch.float32), None,
                      z(2, 5, dtype=torch.float32), z(2, 4), z(2), z(2))
    with pytest.raises(ValueError):
        B.kv_append(params(), shape(), t, z(2, 4, 4, 64, dtype=bf), z(2, 4, 4, 64, dtype=bf), k, k,
                    B.kv_layout(k))
    with pytest.raises(ValueError):
        B.make_tree(300, PTR, plan=z(1))


def test_a_tree_keeps_its_tensors():
    """Its tensors cannot be exchanged under the pointers that it holds."""
    t = B.make_tree(4, PTR)
    for name in ("nodes", "base", "count", "plan"):
        with pytest.raises(AttributeError):
            setattr(t, name, None)
    assert (t.nodes, t.base, t.count, t.plan) == (4, PTR, None, None)


def test_plan_needs_a_buffer():
    with pytest.raises(ValueError):
        B.tree_plan(torch.zeros((2, 4), dtype=torch.int32), None, None)


def test_layouts_know_how_many_scales_they_hold():
    """A layout of one layer's scales is not one for an append of several layers."""
    lay = B.kv_layout(torch.zeros((2, 4, 120, 64), dtype=torch.uint8))
    B._need_extents(lay, 2, 4, 1000)  # none: nothing is read
    lay.scales, lay.bases = 8, 2
    B._need_extents(lay, 2, 4)
    B._need_extents(lay, 1, 4, 2)
    for wrong in ((2, 4, 2), (3, 4), (2, 8)):
        with pytest.raises(ValueError):
            B._need_extents(lay, *wrong)
    lay.scales = 1 << 20
    with pytest.raises(ValueError):
        B._need_extents(lay, 3, 4)


@pytest.mark.parametrize("heads", [1, 4, 20, 32, 64])
def test_few_tiles_per_wave_stay_whole(heads):
    """Up to three of d = 64 and two of d = 128, whatever the number of heads."""
    for d, most in ((64, 24), (128, 16)):
        for tiles in range(4, 60):
            keys = (tiles - 2) * 32  # two more where lists end inside a tile
            for more in (0, -31):
                p = params(prompt_len=keys + more - 7 - 4, grid_h=2, grid_w=2)
                i = B.tree_launch_info(p, shape(1, heads, heads, d), 7)
                assert (i.splits == 1) == (tiles <= most), (d, tiles)
