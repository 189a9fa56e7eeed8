"""Refusals and sizes of the calls over pages and of the beam selection, on the host:
nothing is launched."""

import ctypes as C

import pytest
import torch

from paper_2609_19702_amd import binding as B

P0 = B.make_params(32, 16, 16, 64, 13, B.MODE_DENSE)
PD = B.make_params(32, 16, 16, 64, 13, B.MODE_DIAGONAL)
S0 = B.make_shape(2, 8, 8, 64)
AT = 1 << 20  # an aligned address that is never read


def pages(**kw):
    f = dict(page_rows=16, max_pages=18, num_pages=40, d_table=AT, d_refs=AT, d_cursor=AT,
             d_prompt=None)
    f.update(kw)
    return B.PagesStruct(**f)


def layout(**kw):
    f = dict(num_pages=40, page_rows=16, stride_page=8 * 16 * 64, stride_head=16 * 64, stride_row=64,
             d_k_scale=None, d_v_scale=None, dtype=B.KV_BF16)
    f.update(kw)
    return B.PageLayout(**f)


BAD_PAGES = [dict(page_rows=0), dict(page_rows=3), dict(page_rows=2048), dict(page_rows=-8),
             dict(max_pages=0), dict(max_pages=1 << 27), dict(d_table=None)]
BAD_POOL = [dict(num_pages=0), dict(num_pages=1 << 27), dict(d_refs=None)]


def update(p=P0, batch=2, g=None, length=AT, new=None, most=4, slots=AT, pos=AT, copies=AT,
           flags=AT):
    g = pages() if g is None else g
    return B.lib().dsa_page_update(C.byref(p), batch, C.byref(g), length, new, most, slots, pos,
                                   copies, flags, None)


@pytest.mark.parametrize("bad", [dict(batch=0), dict(length=None), dict(most=0), dict(slots=None),
                                 dict(pos=None), dict(copies=None), dict(flags=None),
                                 dict(batch=4096, most=1 << 20),
                                 dict(p=B.make_params(32, 16, 16, 0, 13))]
                         + [dict(g=pages(**x)) for x in BAD_PAGES + BAD_POOL
                            + [dict(d_cursor=None)]])
def test_update_refuses(bad):
    assert update(**bad) == B.ERR_INVALID_ARG


def test_update_refuses_large_batches():
    assert update(batch=B.MAX_PAGED_BATCH + 1) == B.ERR_UNSUPPORTED


def test_reorder_refuses():
    def call(batch=2, g=None, parent=AT):
        g = pages() if g is None else g
        return B.lib().dsa_page_reorder(batch, C.byref(g), parent, None)

    assert call(batch=0) == call(parent=None) == B.ERR_INVALID_ARG
    assert call(batch=B.MAX_PAGED_BATCH + 1) == B.ERR_UNSUPPORTED
    for x in BAD_PAGES + BAD_POOL:
        assert call(g=pages(**x)) == B.ERR_INVALID_ARG
    assert B.lib().dsa_page_reorder(2, None, AT, None) == B.ERR_INVALID_ARG


BAD_LAYOUT = [dict(num_pages=0), dict(page_rows=12), dict(num_pages=1 << 27), dict(stride_page=-8),
              dict(stride_head=4), dict(stride_row=-64), dict(d_k_scale=AT),
              dict(dtype=B.KV_FP8_E4M3, stride_row=72), dict(dtype=2), dict(dtype=-1)]


def append(s=S0, most=1, slots=AT, kn=AT, vn=AT, rows=(1024, 1024, 64, 0), layers=1, k=AT, v=AT,
           l=None, stride=0, copies=None):
    l = layout() if l is None else l
    rows = None if rows is None else C.byref(B.NodeRows(*rows))
    return B.lib().dsa_paged_append(C.byref(s), most, slots, kn, vn, rows, layers, k, v, C.byref(l),
                                    stride, copies, None)


@pytest.mark.parametrize("bad", [dict(most=0), dict(slots=None), dict(kn=None), dict(vn=None),
                                 dict(kn=AT + 8), dict(rows=None), dict(rows=(1024, 1024, 60, 0)),
                                 dict(rows=(-8, 1024, 64, 0)), dict(layers=0), dict(k=None),
                                 dict(v=AT + 2), dict(stride=4), dict(stride=-8),
                                 dict(layers=1 << 30), dict(most=1 << 30),
                                 dict(stride=8, l=layout(dtype=B.KV_FP8_E4M3)),
                                 dict(s=B.make_shape(0, 8, 8, 64))]
                         + [dict(l=layout(**x)) for x in BAD_LAYOUT])
def test_append_refuses(bad):
    assert append(**bad) == B.ERR_INVALID_ARG


def test_unsupported_shapes():
    assert append(s=B.make_shape(2, 8, 8, 96)) == B.ERR_UNSUPPORTED
    assert attend(s=B.make_shape(2, 24, 8, 64)) == B.ERR_UNSUPPORTED


def attend(p=P0, s=S0, g=None, q=AT, k=AT, v=AT, l=None, pos=AT, plan=None, scale=0.1, out=AT,
           kind=0, logits=None, ws=AT, ws_bytes=1 << 40):
    g, l = pages() if g is None else g, layout() if l is None else l
    return B.lib().dsa_paged_attention(C.byref(p), C.byref(s), C.byref(g), q, k, v, C.byref(l), pos,
                                       plan, scale, out, kind, logits, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=AT + 8), dict(k=None), dict(v=AT + 1),
                                 dict(pos=None), dict(out=None), dict(out=AT + 4), dict(kind=2),
                                 dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(logits=AT), dict(p=PD), dict(g=pages(page_rows=32)),
                                 dict(p=B.make_params(-1, 16, 16, 64, 13))]
                         + [dict(g=pages(**x)) for x in BAD_PAGES]
                         + [dict(l=layout(**x)) for x in BAD_LAYOUT])
def test_attention_refuses(bad):
    assert attend(**bad) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [2.0 ** 126 * 1.0001, -2.0 ** 127, 3e38])
def test_attention_refuses_scales_whose_scores_would_overflow(scale):
    assert attend(scale=scale) == B.ERR_INVALID_ARG


def test_attention_asks_for_its_workspace():
    p, s = B.make_params(32, 64, 64, 64, 13, B.MODE_DENSE), B.make_shape(1, 8, 8, 128)
    g = pages(max_pages=300)
    need = B.paged_workspace_bytes(p, s)
    assert need > 0
    assert attend(p, s, g, ws=None) == attend(p, s, g, ws_bytes=need - 1) == B.ERR_WORKSPACE
    assert attend(p, s, g, ws=AT + 4, ws_bytes=need) == B.ERR_INVALID_ARG
    bad = B.make_params(32, 0, 64, 64, 13, B.MODE_DENSE)
    assert B.paged_workspace_bytes(bad, s) == 0
    with pytest.raises(B.DSAError):
        B.paged_launch_info(bad, s)


@pytest.mark.parametrize("mode", [B.MODE_DENSE, B.MODE_DIAGONAL, B.MODE_WINDOW])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64), (1, 20, 20, 64), (128, 32, 32, 128), (3, 32, 4, 128),
                                   (700, 8, 8, 64)])
def test_launches_cover_all_rows(mode, shape):
    for prompt, grid in ((0, (1, 1)), (120, (24, 24)), (256, (96, 96)), (1 << 20, (4096, 4096))):
        p, s = B.make_params(prompt, *grid, 64, 13, mode), B.make_shape(*shape)
        if B.validate(p, s) != B.OK:
            continue
        rows = prompt + (grid[0] * grid[1] if mode == B.MODE_DENSE else min(13, grid[0] * grid[1]))
        i = B.paged_launch_info(p, s)
        assert i.rows_per_split % 64 == 0 and i.rows_per_split <= 896 and i.waves_per_group == 8
        assert i.max_splits * i.rows_per_split >= rows > (i.max_splits - 1) * i.rows_per_split
        assert i.workgroups == shape[0] * shape[2] * i.max_splits
        assert (i.workspace_bytes > 0) == (i.max_splits > 1)
        assert i.workspace_bytes == B.paged_workspace_bytes(p, s)


def beam(batch=2, beams=4, vocab=100, x=AT, stride=100, kind=0, score=AT, nxt=AT, parent=AT,
         token=AT, ws=AT, ws_bytes=1 << 40):
    return B.lib().dsa_beam_select(batch, beams, vocab, x, stride, kind, score, nxt, parent, token,
                                   ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(batch=0), dict(beams=0), dict(beams=B.MAX_BEAMS + 1),
                                 dict(vocab=0), dict(vocab=(1 << 24) + 1, stride=1 << 25),
                                 dict(batch=1 << 20), dict(x=None), dict(stride=99), dict(kind=2),
                                 dict(score=None), dict(nxt=None), dict(parent=None),
                                 dict(token=None), dict(ws=AT + 8)])
def test_beam_refuses(bad):
    assert beam(**bad) == B.ERR_INVALID_ARG


def test_beam_asks_for_its_workspace():
    need = B.beam_workspace_bytes(2, 4, 100)
    assert need > 0 and B.beam_workspace_bytes(2, 17, 100) == 0
    assert beam(ws=None) == beam(ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_binding_refuses():
    """CPU tensors, and what does not fit together."""
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        B.make_pages(16, i32(2, 4))
    k = torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16)
    assert B.page_layout(k).num_pages == 5 and B.page_layout(k).page_rows == 16
    with pytest.raises(ValueError, match="contiguous"):
        B.page_layout(k.transpose(2, 3))
    with pytest.raises(ValueError, match="num_pages"):
        B.page_layout(k[0])
    with pytest.raises(ValueError, match="dtype"):
        B.page_layout(k.float())
    with pytest.raises(ValueError, match="GPU"):
        B.page_layout(k.to(torch.float8_e4m3fn), torch.ones(2))
    x = torch.zeros((2, 4, 100))
    with pytest.raises(ValueError, match="must be"):
        B.beam_select(x[0], *[None] * 5)
    with pytest.raises(ValueError, match="fp32 or bf16"):
        B.beam_select(x.half(), *[None] * 5)


def test_a_changed_layout_is_looked_at_again():
    s, k = B.make_shape(2, 8, 8, 64), torch.zeros(40, 8, 16, 64, dtype=torch.bfloat16)
    at = B.page_layout(k)
    for _ in range(2):
        B._check_paged(s, k, k, at, None, k.get_device())
    at.num_pages = 41
    with pytest.raises(ValueError, match="does not hold 41 pages"):
        B._check_paged(s, k, k, at, None, k.get_device())
    at.num_pages, at.stride_row = 40, 128
    with pytest.raises(ValueError, match="does not hold"):
        B._check_paged(s, k, k, at, None, k.get_device())
    at.stride_row = 64
    B._check_paged(s, k, k, at, None, k.get_device())
    with pytest.raises(ValueError, match="does not hold"):
        B._check_paged(s, k[:39], k[:39], at, None, k.get_device())
