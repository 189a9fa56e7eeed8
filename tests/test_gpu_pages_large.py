"""Tables and pools of the largest sizes that the calls take: places of 31 bits."""

import pytest
import torch

from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, ints

pytestmark = pytest.mark.gpu

MOST = (1 << 31) - 1


def filled(n, value):
    return torch.full((n,), value, dtype=torch.int32, device=DEV)


class Pool:
    """Two requests over a pool of one-row pages."""

    def __init__(self, refs, cursor, width=8):
        self.p = B.make_params(0, 64, 64, 1, 1, B.MODE_DENSE)
        self.pages = B.make_pages(1, torch.full((2, width), -1, dtype=torch.int32, device=DEV), refs,
                                  ints([cursor]))
        self.slots = torch.full((2, width), 7, dtype=torch.int32, device=DEV)
        self.pos, self.flags = ints([7, 7]), ints([7, 7])
        self.copies = torch.full((2, 3), 7, dtype=torch.int32, device=DEV)

    def update(self, lengths, new):
        B.page_update(self.p, self.pages, ints(lengths), ints(new), self.slots, self.pos,
                      self.copies, self.flags)
        return self.flags.tolist()


@pytest.mark.parametrize("pool,cursor", [(MOST, MOST - 1), (MOST, MOST - 3), (MOST, 1 << 30),
                                         (MOST, -2), (MOST, MOST), (MOST - 4095, MOST - 4096),
                                         ((1 << 30) + 1, 1 << 30), ((1 << 30) + 4099, (1 << 30) + 7)])
def test_a_large_pool_is_searched_around(pool, cursor):
    """From the cursor on, past the pool's end to its beginning."""
    refs = filled(pool, 0)
    start = cursor % pool if cursor >= 0 else (cursor + pool) % pool
    busy = [(start + i) % pool for i in (0, 2, 5)]
    refs[torch.tensor(busy, device=DEV)] = 9
    free = [(start + i) % pool for i in range(12) if i not in (0, 2, 5)]
    x = Pool(refs, cursor)
    assert x.update([0, 0], [4, 3]) == [0, 0]
    assert x.slots.tolist() == [free[:4] + [-1] * 4, free[4:7] + [-1] * 5]
    assert x.pages.table.tolist() == x.slots.tolist()
    assert x.pages.cursor.item() == (free[6] + 1) % pool
    at = torch.tensor(free[:7], device=DEV)
    assert (refs[at] == 1).all() and (refs[torch.tensor(busy, device=DEV)] == 9).all()
    refs[at] = 0
    refs[torch.tensor(busy, device=DEV)] = 0
    assert not refs.any()


@pytest.mark.parametrize("pool", [MOST, (1 << 30) + 3])
def test_the_last_pages_that_a_large_pool_is_searched_for(pool):
    """All but the two before the cursor, and one at the pool's end, are taken."""
    refs = filled(pool, 1)
    cursor = (1 << 30) - 5
    refs[pool - 1] = refs[cursor - 1] = refs[cursor - 2] = 0
    x = Pool(refs, cursor)
    assert x.update([0, 0], [1, 2]) == [0, 0]
    assert x.pages.table[:, :2].tolist() == [[pool - 1, -1], [cursor - 2, cursor - 1]]
    assert x.pages.cursor.item() == cursor
    assert (refs == 1).all()
    assert x.update([1, 2], [1, 1]) == [1, 1]  # none is left
    assert x.slots.tolist() == [[-1] * 8] * 2 and x.pages.cursor.item() == cursor


@pytest.mark.parametrize("batch,width", [(1, MOST), (2, MOST // 2), (1, MOST - 15), (3, 70000001),
                                         (130, 9000001)])
def test_long_rows_of_a_table(batch, width):
    """More columns than a launch has workgroups for, the last ones of 31 bits."""
    g = torch.Generator(device=DEV).manual_seed(1)
    table = torch.empty((batch, width), dtype=torch.int32, device=DEV)
    table.fill_(-1)
    at = torch.randint(0, width, (batch, 5000), generator=g, device=DEV)
    at[:, :3] = torch.tensor([0, width - 1, width - 2], device=DEV)
    table.scatter_(1, at, torch.randint(0, 100, at.shape, generator=g, device=DEV,
                                        dtype=torch.int32))
    refs = filled(100, 1 << 20)
    pages = B.make_pages(1, table, refs)
    for parent in ([batch - 1 - b for b in range(batch)], [-1] + [0] * (batch - 1)):
        want = torch.full((batch, 5000), -1, dtype=torch.int32, device=DEV)
        here = torch.stack([table[p].gather(0, at[b]) if p >= 0 else want[b]
                            for b, p in enumerate(parent)])
        count = [int((table[p] >= 0).sum()) if p >= 0 else 0 for p in parent]
        users = torch.zeros(100, dtype=torch.int64, device=DEV)
        for p in parent:
            if p >= 0:
                users += torch.bincount(table[p][table[p] >= 0], minlength=100)
        for b in range(batch):
            users -= torch.bincount(table[b][table[b] >= 0], minlength=100)
        before = refs.long()
        B.page_reorder(pages, ints(parent))
        assert torch.equal(table.gather(1, at), here)
        assert [int((table[b] >= 0).sum()) for b in range(batch)] == count
        assert torch.equal(refs.long(), before + users)


@pytest.mark.parametrize("page,width", [(1, MOST), (1, MOST - 1), (2, MOST // 2), (16, MOST // 16)])
def test_the_last_rows_of_the_longest_table(page, width):
    """Requests of close to 2^31 rows, with few and many slots."""
    table = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    p = B.make_params(0, 64, 64, 1, 1, B.MODE_DENSE)
    for most in (1, 16, 17, 65):
        for new in {1, 3, most}:
            new = min(new, most)
            length = width * page - new
            entries = list(range(length // page, width))
            refs = filled(100, 0)
            pages = B.make_pages(page, table, refs, ints([7]))
            slots = torch.full((1, most), 7, dtype=torch.int32, device=DEV)
            pos, copies, flags = ints([7]), ints([[7, 7, 7]]), ints([7])

            def update(at, n):
                B.page_update(p, pages, ints([at]), ints([n]), slots, pos, copies, flags)

            update(length, new)
            got = [7 + i for i in range(len(entries))]
            assert table[0, entries[0]:].tolist() == got and flags.item() == 0
            assert pos.item() == length + new - 1 and copies.tolist() == [[-1] * 3]
            want = [got[r // page - entries[0]] * page + r % page
                    for r in range(length, length + new)]
            assert slots.tolist() == [want + [-1] * (most - new)]
            assert refs.nonzero().view(-1).tolist() == got and (refs <= 1).all()
            update(length, new + 1)  # clamped to the slots, or a row too many
            assert flags.item() == (B.PAGE_FLAG_TOO_LONG if new < most else 0)
            update(MOST, 1)
            assert flags.item() == B.PAGE_FLAG_TOO_LONG
            update(width * page, 0)
            assert flags.item() == 0 and slots.tolist() == [[-1] * most]
            table[0, entries[0]:] = -1
    assert not (table != -1).any()


def test_slots_past_31_bits_of_bytes():
    """As many slots as a call takes: those past the new rows hold -1."""
    most = MOST
    slots = torch.full((1, most), 7, dtype=torch.int32, device=DEV)
    table = torch.full((1, 9), -1, dtype=torch.int32, device=DEV)
    pos, copies, flags = ints([7]), ints([[7, 7, 7]]), ints([7])
    p = B.make_params(0, 64, 64, 1, 1, B.MODE_DENSE)
    B.page_update(p, B.make_pages(4, table, filled(9, 0), ints([0])), ints([0]), ints([30]), slots,
                  pos, copies, flags)
    assert slots[0, :30].tolist() == list(range(30)) and (slots[0, 30:] == -1).all()
