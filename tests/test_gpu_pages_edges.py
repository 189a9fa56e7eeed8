"""Corners of the calls over pages: scales of any kind, pools with not a page to spare, plans with
rows out of range."""

import math

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, Attend
from tests.test_gpu_pages import Append, Tables, e4m3, users

pytestmark = pytest.mark.gpu

ONES = 2 - 2.0 ** -23  # a mantissa of ones
SCALES = [1.0, -1.0, -0.37, 0.37, ONES, ONES / 2, -ONES * 2.0 ** -9, ONES * 2.0 ** -7, 1 + 2.0 ** -23,
          1.9999, 448.0, 3.0, 1 / 3, 2.0 ** -79, ONES * 2.0 ** -80, 2.0 ** -80, 2.0 ** -90, 2.0 ** 79,
          ONES * 2.0 ** 79, 2.0 ** 80, -2.0 ** 90, ONES * 2.0 ** 127, 2.0 ** -126, 1e-40, 2.0 ** -149,
          0.0, -0.0, math.inf, -math.inf, math.nan]


def test_append_divides_by_scales_of_any_kind():
    """Every bf16 value over each of them, a KV head each: the codes of the division rounded to
    fp32, as on the CPU."""
    g = torch.Generator().manual_seed(1)
    more = (1 + torch.rand(2 * 40 - len(SCALES), generator=g)) * 2.0 ** torch.randint(
        -12, 12, (2 * 40 - len(SCALES),), generator=g)
    scales = torch.cat([torch.tensor(SCALES, dtype=torch.float64).float(), more.float()])
    x = Append(layers=1, batch=1, n=512, hkv=40, d=128, page=128, pool=10, kv="fp8", copies=False)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(512, 128).view(torch.bfloat16)
    x.new[0, 0] = bits[:, None].expand(512, 80, 128).to(DEV)
    x.ks, x.vs = (s.view(1, 40).contiguous().to(DEV) for s in scales.split(40))
    x.slots = [[(37 * i) % 1280 for i in range(512)]]
    x.run()
    at = torch.tensor(x.slots[0])
    new = bits.float()
    for i, s in enumerate(scales.tolist()):
        t = (x.k, x.v)[i // 40].view(torch.uint8)[0, :, i % 40].reshape(-1, 128)[at].cpu()
        div = new / torch.tensor(s)
        want = e4m3(new, torch.full_like(new, s)).view(torch.uint8)
        nan = div.isnan()
        assert torch.equal(t[~nan], want[~nan]), s
        assert ((t[nan] & 127) == 127).all(), s


def test_a_page_that_its_last_users_leave_is_free_only_in_the_next_call():
    t = Tables(3, 4, 3, pool=3, most=2, prompt=0)
    t.step([0, -1, -1], [1, 0, 0])
    t.reorder([0, 0, -1])
    # two leave the page that they share for the two free ones; the third needs one
    _, _, _, flags = t.step([1, 1, 0], [1, 1, 2])
    assert flags == [0, 0, B.PAGE_FLAG_NO_PAGES] and t.refs == [0, 1, 1]
    assert t.table == [[1, -1, -1], [2, -1, -1], [-1, -1, -1]]
    _, _, _, flags = t.step([2, 2, 0], [1, 1, 2])
    assert flags == [0, 0, 0] and t.table[2] == [0, -1, -1] and users(t) == t.refs


def test_who_gets_no_page_keeps_the_shared_one():
    t = Tables(3, 4, 3, pool=3, most=1, prompt=0)
    t.step([0, -1, -1], [1, 0, 0])
    t.reorder([0, 0, 0])
    _, pos, copies, flags = t.step([1, 1, 1], [1, 1, 1])
    assert flags == [0, 0, B.PAGE_FLAG_NO_PAGES] and copies == [[0, 1, 1], [0, 2, 1], [-1] * 3]
    assert t.table[2] == [0, -1, -1] and t.refs == [1, 1, 1] and pos[2] == -1
    # it is the only user now, and writes where it is
    slots, _, copies, flags = t.step([2, 2, 1], [1, 1, 1])
    assert flags == [0, 0, 0] and slots[2] == [1] and copies[2] == [-1] * 3 and t.refs == [1, 1, 1]


@pytest.mark.parametrize("group", [1, 4])
def test_a_corrupt_plan_is_the_clamped_one(group):
    """Places below 0 and past the step's position, and counts below 0 and past the list."""
    x = Attend(batch=2, heads=(2 * group, 2), mode="diagonal", n_att=10, window=20, pos=[50, 60],
               page=8, hidden=0.5, seed=3)
    count, _, places = B.plan_views(x.p, x.s, x.plan)
    whole = [count.clone(), places.clone()]

    def run(bad):
        count.copy_(whole[0])
        places.copy_(whole[1])
        if bad:
            places[0, 0], places[0, 1], places[3, 9] = -7, 1 << 30, -(1 << 31)
            count[1], count[2] = 1 << 20, -5
        else:
            places[0, 0], places[0, 1], places[3, 9] = 0, 50, 0
            count[1], count[2] = 10, 0
        x.out.fill_(7.0)
        x.logits.fill_(7.0)
        x.run()
        return x.out.clone(), x.logits.clone()

    assert all(torch.equal(p, q) for p, q in zip(run(True), run(False)))
    assert x.out.isfinite().all()
