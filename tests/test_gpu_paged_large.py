"""Appends and attention over pages with more workgroups than a launch holds: the last
ones do their work too."""

import math

import numpy as np
import pytest
import torch

from oracle import paged as opaged
from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, ints

pytestmark = pytest.mark.gpu

THREADS = 1 << 32  # a launch has fewer


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_rows_of_many_requests_and_layers(kv):
    """A table of 4096 slots, a few of them in use, prompts into all layers at once."""
    layers, batch, hkv, d, page = 33, 4096, 32, 128, 16
    n = 64 if kv == "bf16" else 128
    chunks = hkv * d * (2 if kv == "bf16" else 1) // 16
    assert layers * batch * (n * chunks // 256) * 256 >= THREADS
    k = torch.zeros((layers, 6, hkv, page, d), device=DEV).bfloat16()
    k = k if kv == "bf16" else k.to(torch.float8_e4m3fn)
    v = torch.zeros_like(k)
    rows = torch.randn((layers, 1, n, 2 * hkv, d), device=DEV).bfloat16()
    slots = torch.full((batch, n), -1, dtype=torch.int32, device=DEV)
    used = [(0, 3, 5), (0, n - 1, 17), (2000, 0, 40), (4094, 7, 50), (4095, 0, 70), (4095, n - 1, 95)]
    for b, i, slot in used:
        slots[b, i] = slot
    new = rows.expand(layers, batch, n, 2 * hkv, d)
    B.paged_append(B.make_shape(batch, hkv, hkv, d), slots, new[:, :, :, :hkv], new[:, :, :, hkv:],
                   k, v, B.page_layout(k[0]))
    for t, x in ((k, rows[:, 0, :, :hkv]), (v, rows[:, 0, :, hkv:])):
        want = torch.zeros((layers, 6, hkv, page, d), device=DEV)
        for b, i, slot in used:
            want[:, slot // page, :, slot % page] = x[:, i].to(t.dtype).float()
        assert torch.equal(t.float(), want)


def test_copies_of_many_requests():
    layers, batch, hkv, d, page = 2, 4096, 32, 128, 1024
    assert layers * batch * (2 + page * hkv * d * 2 // 16 // 256) * 256 >= THREADS
    k = torch.randn((layers, 4, hkv, page, d), device=DEV).bfloat16()
    v = torch.randn((layers, 4, hkv, page, d), device=DEV).bfloat16()
    want = [t.clone() for t in (k, v)]
    copies = torch.full((batch, 3), -1, dtype=torch.int32, device=DEV)
    copies[3], copies[4095] = ints([0, 1, 1024]), ints([2, 3, 777])
    for t in want:
        t[:, 1] = t[:, 0]
        t[:, 3, :, :777] = t[:, 2, :, :777]
    new = torch.zeros((1, 1, 1, hkv, d), device=DEV).bfloat16().expand(layers, batch, 1, hkv, d)
    slots = torch.full((batch, 1), -1, dtype=torch.int32, device=DEV)
    B.paged_append(B.make_shape(batch, hkv, hkv, d), slots, new, new, k, v, B.page_layout(k[0]), copies)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("group", [1, 2])
def test_splits_of_many_requests(group):
    """Two hundred requests of up to 2^25 rows each, one of which is that long; most of
    its entries name no page.  The bound is that of ``Attend.check``: what is added for
    splits without rows is 0."""
    batch, d, page, prompt = 200, 64, 1024, 1 << 24
    p = B.make_params(prompt, 4096, 4096, 1, 1, B.MODE_DENSE)
    s = B.make_shape(batch, group, 1, d)
    assert B.paged_launch_info(p, s).workgroups * 512 >= THREADS
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((4, 1, page, d), generator=g).bfloat16() for _ in range(2))
    q = torch.randn((batch, group, d), generator=g).bfloat16()
    table = torch.full((batch, 1 << 15), -1, dtype=torch.int32)
    long, short = 123, {0: 40, 55: 1000, 199: 3}
    table[long, 5], table[long, -2], table[long, -1] = 0, 3, 1
    pos, front = torch.full((batch,), -1, dtype=torch.int32), torch.zeros(batch, dtype=torch.int32)
    pos[long], front[long] = (1 << 24) - 1, prompt
    for b, n in short.items():
        table[b, 0], pos[b] = 2, n - 1
    pages = B.make_pages(page, table.to(DEV), prompt=front.to(DEV))
    kd, vd, out = k.to(DEV), v.to(DEV), torch.full((batch, group, d), 7.0, device=DEV)
    ws = torch.empty(B.paged_workspace_bytes(p, s), dtype=torch.uint8, device=DEV)
    B.paged_attention(p, s, pages, q.to(DEV), kd, vd, B.page_layout(kd), pos.to(DEV), 1 / math.sqrt(d),
                      out, workspace=ws)
    out, u = out.double().cpu().numpy(), 2.0 ** -24
    for b in range(batch):
        if b not in short and b != long:
            assert (out[b] == 0).all()
            continue
        at = [0, 3, 1] if b == long else [2]
        n = page if b == long else short[b]
        kb, vb = (x[at, 0, :n].double().numpy().reshape(-1, d) for x in (k, v))
        for h in range(group):
            qh = q[b, h].double().numpy()
            want, _, mass = opaged.attention(qh, kb, vb, 1 / math.sqrt(d))
            dz = (np.abs(kb) @ np.abs(qh)).max() / math.sqrt(d) * (d + 4) * u
            bound = (2 * dz + 4 * u + (2 * len(kb) + 64) * u) * mass + u * np.abs(want) + 1e-30
            assert (np.abs(out[b, h] - want) <= bound).all(), (b, h)
