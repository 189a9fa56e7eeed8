"""Page tables from request lengths, and tables reordered, against the sequential
reference; appends into pages, bit for bit."""

import random

import pytest
import torch

from oracle import paged as opaged
from paper_2609_19702_amd import binding as B
from tests.paged_util import DEV, MODES, ints

pytestmark = pytest.mark.gpu


class Tables:
    """Tables on the GPU beside the reference's."""

    def __init__(self, batch, page, width, pool, most, mode="dense", prompt=20, prompts=None,
                 sinks=0, n_att=1, window=1, cursor=0):
        self.page, self.most = page, most
        self.p = B.make_params(prompt, 64, 64, window, n_att, MODES[mode], sinks)
        self.sinks = 0 if mode == "dense" else sinks
        self.window = {"dense": 0, "window": n_att - sinks, "diagonal": window}[mode]
        self.front = [min(max(x, 0), prompt) for x in prompts] if prompts else [prompt] * batch
        self.table, self.refs, self.cursor = [[-1] * width for _ in range(batch)], [0] * pool, cursor
        self.pages = B.make_pages(page, ints(self.table), ints(self.refs), ints([cursor]),
                                  ints(prompts) if prompts else None)
        self.slots = torch.full((batch, most), 7, dtype=torch.int32, device=DEV)
        self.pos, self.flags = ints([7] * batch), ints([7] * batch)
        self.copies = torch.full((batch, 3), 7, dtype=torch.int32, device=DEV)

    def put(self):
        """The reference's tables onto the GPU."""
        self.pages.table.copy_(ints(self.table))
        self.pages.refs.copy_(ints(self.refs))
        self.pages.cursor.copy_(ints([self.cursor]))

    def issue(self, lengths, new, stream=None):
        B.page_update(self.p, self.pages, lengths, new, self.slots, self.pos, self.copies,
                      self.flags, stream=stream)

    def expect(self, lengths, new):
        got = opaged.update(self.table, self.refs, self.cursor, self.front, lengths, new, self.most,
                            self.page, self.sinks, self.window)
        self.cursor = got[0]
        return got[1:]

    def check(self, want):
        assert self.pages.table.tolist() == self.table
        assert self.pages.refs.tolist() == self.refs
        assert self.pages.cursor.tolist() == [self.cursor]
        for x, y in zip((self.slots, self.pos, self.copies, self.flags), want):
            assert x.tolist() == y

    def step(self, lengths, new, null=False):
        want = self.expect(lengths, new)
        self.issue(ints(lengths), None if null else ints(new))
        self.check(want)
        return want

    def reorder(self, parent):
        self.table = opaged.reorder(self.table, self.refs, parent)
        B.page_reorder(self.pages, ints(parent))
        assert self.pages.table.tolist() == self.table
        assert self.pages.refs.tolist() == self.refs


def users(t):
    """How many entries name each page."""
    n = [0] * len(t.refs)
    for line in t.table:
        for e in line:
            if e >= 0:
                n[e] += 1
    return n


@pytest.mark.parametrize("mode,sinks", [("dense", 0), ("window", 0), ("window", 4), ("diagonal", 4)])
@pytest.mark.parametrize("batch,page", [(1, 16), (5, 1), (17, 8), (70, 16), (33, 64)])
def test_requests_come_go_and_share(mode, sinks, batch, page):
    """Steps of a serving loop against the reference, and every page with as many
    users as its count says."""
    rng = random.Random(batch * page)
    width, prompts = 300 // page + 2, [rng.randrange(0, 41) for _ in range(batch)]
    t = Tables(batch, page, width, pool=batch * width * 2 // 3 + 5, most=50, mode=mode, prompt=40,
               prompts=prompts, sinks=sinks, n_att=sinks + 30, window=60, cursor=7)
    length = [-1] * batch
    copied = 0
    for i in range(40):
        new = []
        for b in range(batch):
            if length[b] < 0 or rng.random() < 0.05:
                length[b] = rng.choice([-1, 0, 0])
            new.append(prompts[b] if length[b] == 0 else rng.choice([1, 1, 1, 0, 7, 50]))
        if i % 3 == 2:
            parent = [rng.randrange(-1, batch) if rng.random() < 0.3 else b for b in range(batch)]
            t.reorder(parent)
            length = [length[p] if p >= 0 else -1 for p in parent]
            prompts = [prompts[p] if p >= 0 else prompts[b] for b, p in enumerate(parent)]
            new = [new[p] if p >= 0 else 0 for p in parent]
            t.front = list(prompts)
            t.pages.prompt.copy_(ints(prompts))
        _, pos, copies, flags = t.step(length, new)
        assert users(t) == t.refs
        copied += sum(c[0] >= 0 for c in copies)
        for b in range(batch):
            if flags[b]:
                length[b] = -1  # a program lets it go
            elif length[b] >= 0:
                length[b] += min(new[b], 50)
                if rng.random() < 0.1:
                    length[b] -= rng.randrange(0, min(9, length[b] + 1))  # drafts not taken
    assert batch < 17 or copied


def test_a_pool_that_runs_short():
    rng = random.Random(4)
    t = Tables(40, 8, 20, pool=150, most=30, prompt=0)
    at, short = [0] * 40, 0
    for i in range(40):
        new = [rng.choice([0, 1, 5, 30]) for _ in at]
        _, _, _, flags = t.step(at, new)
        assert users(t) == t.refs
        short += sum(flags)
        at = [rng.choice([x, -1]) if f else x + n if x >= 0 else 0
              for x, n, f in zip(at, new, flags)]
        at = [-1 if x > 130 else x for x in at]
    assert short > 100


def test_exact_pages():
    """A worked case: the cursor, its way around, and requests in order."""
    t = Tables(3, 4, 5, pool=8, most=6, prompt=0, cursor=6)
    slots, pos, _, flags = t.step([0, 0, 0], [6, 4, 5])
    assert t.table == [[6, 7, -1, -1, -1], [0, -1, -1, -1, -1], [1, 2, -1, -1, -1]]
    assert slots == [[24, 25, 26, 27, 28, 29], [0, 1, 2, 3, -1, -1], [4, 5, 6, 7, 8, -1]]
    assert pos == [5, 3, 4] and flags == [0, 0, 0] and t.cursor == 3
    _, pos, _, flags = t.step([6, 4, 5], [6, 6, 1])  # needs 1, 2 and 0 of pages 3, 4, 5
    assert t.table == [[6, 7, 3, -1, -1], [0, 4, 5, -1, -1], [1, 2, -1, -1, -1]]
    _, pos, _, flags = t.step([12, 10, 6], [2, 2, 6])  # nothing is free
    assert flags == [1, 0, 1] and pos == [-1, 11, -1]
    _, _, _, flags = t.step([-1, 12, 6], [0, 6, 6])  # what leaves can be taken at once
    assert flags == [0, 0, 0] and t.table[1] == [0, 4, 5, 6, 7] and t.table[2] == [1, 2, 3, -1, -1]


def test_shared_pages_are_left_by_who_writes():
    t = Tables(3, 4, 4, pool=12, most=3, prompt=0)
    t.step([0, -1, -1], [3, 0, 0])
    t.step([3, -1, -1], [3, 0, 0])  # pages 0 and 1, two rows in the second
    t.reorder([0, 0, 0])
    assert t.refs[:2] == [3, 3]
    _, _, copies, _ = t.step([6, 6, 6], [1, 0, 3])
    assert t.table == [[0, 2, -1, -1], [0, 1, -1, -1], [0, 3, 4, -1]]
    assert copies == [[1, 2, 2], [-1, -1, -1], [1, 3, 2]] and t.refs[:2] == [3, 1]
    # at a page's start there is nothing to copy; behind it, entries of drafts
    t.reorder([2, 2, 2])
    _, _, copies, _ = t.step([4, -1, 8], [3, 0, 1])
    assert copies[0] == [-1] * 3 and copies[2] == [-1] * 3
    assert users(t) == t.refs


def test_the_last_users_of_a_page_leave_it_to_the_pool():
    t = Tables(2, 4, 3, pool=4, most=1, prompt=0)
    t.step([0, -1], [1, 0])
    t.reorder([0, 0])
    t.step([1, 1], [1, 1])
    assert t.refs == [0, 1, 1, 0] and t.table == [[1, -1, -1], [2, -1, -1]]
    # a page that is left here cannot be taken here
    t.reorder([0, 0])
    _, _, _, flags = t.step([2, 2], [1, 1])
    assert users(t) == t.refs and flags == [0, 0]


def test_too_long_and_bad_values():
    t = Tables(4, 8, 3, pool=20, most=30, prompt=0)
    _, pos, _, flags = t.step([0, 0, 20, 1 << 30], [24, 25, 5, 1])
    assert flags == [0, 2, 2, 2] and pos == [23, -1, -1, -1]
    t.step([24, 0, 0, 0], [0, -5, 1000, 24])  # no new rows; a count below 0; one past the slots
    t.step([24, 2147483647, 3, -(1 << 31)], [0, 30, 1, 1])
    # entries that name no page are as missing ones
    t.table[0][2], t.table[3][0] = 1 << 30, -77
    t.put()
    t.step([20, -1, -1, -1], [1, 1, 1, 1])


def test_one_new_row_each():
    t = Tables(9, 4, 9, pool=90, most=2, prompt=3)
    for i in range(20):
        t.step([i] * 9, [1] * 9, null=True)
    assert t.pos.tolist() == [16] * 9


def test_cursor_of_any_value():
    for c in (-1, -(1 << 31), (1 << 31) - 1, 11, 23):
        t = Tables(2, 4, 4, pool=11, most=4, prompt=0, cursor=c)
        t.step([0, 0], [4, 4])


@pytest.mark.parametrize("batch", [1024, 1025, 4096])
def test_many_requests(batch):
    rng = random.Random(batch)
    t = Tables(batch, 16, 6, pool=batch * 4, most=40, prompt=0)
    length = [rng.randrange(-1, 50) for _ in range(batch)]
    t.step(length, [rng.randrange(0, 41) for _ in range(batch)])
    t.reorder([rng.randrange(-2, batch + 2) for _ in range(batch)])
    t.step([rng.randrange(-1, 50) for _ in range(batch)], [rng.randrange(0, 41) for _ in range(batch)])
    assert users(t) == t.refs


@pytest.mark.parametrize("page", [1, 2, 16])
@pytest.mark.parametrize("most", [1, 3, 4, 5, 8, 9, 16, 17, 65])
@pytest.mark.parametrize("batch", [64, 65, 128, 129, 300])
def test_few_and_many_slots(batch, most, page):
    """Every number of lanes to a request, with as many slots as lanes and one more."""
    rng = random.Random(batch * most + page)
    width = 120 // page + 1
    t = Tables(batch, page, width, pool=batch * width * 3 // 4, most=most, prompt=9, cursor=3)
    length = [rng.randrange(-1, 30) for _ in range(batch)]
    for i in range(4):
        new = [rng.choice([0, 1, most, most, rng.randrange(most + 1)]) for _ in range(batch)]
        flags = t.step(length, new)[3]
        assert users(t) == t.refs
        length = [-1 if flags[b] or rng.random() < 0.1 else max(n, 0) + (new[b] if n >= 0 else 0)
                  for b, n in enumerate(length)]
        if i == 1:
            parent = [rng.randrange(batch) if rng.random() < 0.2 else b for b in range(batch)]
            t.reorder(parent)
            length = [length[b] for b in parent]


def test_a_long_row_and_a_large_pool():
    t = Tables(3, 16, 2000, pool=50000, most=20000, prompt=0, cursor=49000)
    t.refs[5:40000] = [1] * 39995  # others' pages
    t.put()
    t.step([0, 0, 0], [20000, 7, 12345])
    t.step([20000, 7, -1], [1, 16, 0])


@pytest.mark.parametrize("batch,width", [(1, 1), (1, 300), (3, 17), (64, 33), (513, 70), (4096, 9)])
def test_reorder(batch, width):
    rng = random.Random(batch + width)
    t = Tables(batch, 4, width, pool=100, most=1)
    t.table = [[rng.choice([-1, 100, -9, rng.randrange(100)]) for _ in range(width)]
               for _ in range(batch)]
    t.refs = [500] * 100
    t.put()
    t.reorder([rng.randrange(batch) for _ in range(batch)])
    t.reorder([rng.choice([b, -1, batch, 1 << 30, rng.randrange(batch)]) for b in range(batch)])
    t.reorder([batch - 1 - b for b in range(batch)])


def test_a_captured_step():
    """Reorder and update of a graph, replayed over steps of a loop, with eager work
    between the replays."""
    rng = random.Random(3)
    batch = 12
    t = Tables(batch, 8, 30, pool=200, most=9, mode="window", prompt=9, n_att=30, sinks=2)
    length, new, parent = ints([-1] * batch), ints([0] * batch), ints(list(range(batch)))
    t.issue(length, new)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.page_reorder(t.pages, parent)
        t.issue(length, new)
    t.put()
    at = [0] * batch
    for i in range(25):
        move = [rng.randrange(batch) if rng.random() < 0.2 else b for b in range(batch)]
        at = [at[p] for p in move]
        add = [9 if x == 0 else rng.randrange(0, 4) for x in at]
        t.table = opaged.reorder(t.table, t.refs, move)
        want = t.expect(at, add)
        length.copy_(ints(at))
        new.copy_(ints(add))
        parent.copy_(ints(move))
        g.replay()
        t.check(want)
        at = [x + y for x, y in zip(at, add)]
        at = [0 if x > 220 else x for x in at]


def test_two_pools_at_once():
    """Two updates on two streams, with tables of their own."""
    ts = [Tables(40, 8, 20, pool=900, most=30, prompt=0, cursor=c) for c in (5, 600)]
    args = [(ints([0] * 40), ints([n] * 40)) for n in (29, 30)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t, a, st in zip(ts, args, streams):
        t.issue(*a, stream=st)
    torch.cuda.synchronize()
    for t, a in zip(ts, args):
        t.check(t.expect(*[x.tolist() for x in a]))


# ---- appends ---------------------------------------------------------------------

def codes(x):
    return x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x.view(torch.int16)


def e4m3(x, scale):
    """Codes of x / scale, NaN where it is one."""
    return torch.where(x.isnan(), x, (x / scale).clamp(-448, 448)).to(torch.float8_e4m3fn)


class Append:
    def __init__(self, layers=2, batch=3, n=5, hkv=3, d=64, page=8, pool=40, kv="bf16", copies=True,
                 seed=0, order="page"):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.s = B.make_shape(batch, hkv, hkv, d)
        shape = (layers, pool, hkv, page, d)
        self.k, self.v = (torch.randn(shape, generator=g).to(DEV) for _ in range(2))
        dtype = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
        self.k, self.v = self.k.to(dtype), self.v.to(dtype)
        if order == "head":
            self.k, self.v = (self.spread(x) for x in (self.k, self.v))
        self.ks = self.vs = None
        if kv == "fp8":
            self.ks, self.vs = (torch.rand((layers, hkv), generator=g).to(DEV) * 0.02 + 0.002
                                for _ in range(2))
        free = list(range(pool * page))
        rng.shuffle(free)
        self.copies = None
        if copies:
            pages = rng.sample(range(pool), 2 * batch)
            rows = [[pages[2 * b], pages[2 * b + 1], rng.randrange(0, page + 1)]
                    for b in range(batch)]
            rows[batch // 2] = [-1, -1, -1]
            self.copies = ints(rows)
            free = [x for x in free if x // page not in pages]
        self.slots = [[free.pop() if rng.random() < 0.8 else rng.choice([-1, pool * page, -(1 << 31),
                                                                       (1 << 31) - 1])
                       for _ in range(n)] for _ in range(batch)]
        self.new = torch.randn((layers, batch, n, 2 * hkv, d), generator=g).bfloat16().to(DEV)
        self.hkv, self.page, self.layers = hkv, page, layers

    @staticmethod
    def spread(x):
        """Heads outermost, rows and layers apart."""
        layers, n, h, p, d = x.shape
        y = torch.zeros((layers, h, n + 1, p + 1, d + 16), dtype=torch.float32).to(x.dtype).to(DEV)
        y = y[:, :, :n, :p, :d].permute(0, 2, 1, 3, 4)
        codes(y).copy_(codes(x))
        return y

    def expect(self):
        got = []
        for x, new, s in ((self.k, self.new[:, :, :, :self.hkv], self.ks),
                          (self.v, self.new[:, :, :, self.hkv:], self.vs)):
            x = codes(x).clone()
            if self.copies is not None:
                for a, b, n in self.copies.tolist():
                    if a >= 0:
                        x[:, b, :, :n] = x[:, a, :, :n].clone()
            for b, line in enumerate(self.slots):
                for i, slot in enumerate(line):
                    if 0 <= slot < x.shape[1] * self.page:
                        y = new[:, b, i]
                        if s is not None:
                            y = e4m3(y.float(), s[:, :, None])
                        x[:, slot // self.page, :, slot % self.page] = codes(y)
            got.append(x)
        return got

    def run(self, stream=None):
        B.paged_append(self.s, ints(self.slots), self.new[:, :, :, :self.hkv],
                       self.new[:, :, :, self.hkv:], self.k, self.v,
                       B.page_layout(self.k[0], self.ks, self.vs), self.copies, stream=stream)

    def check(self):
        want = self.expect()
        self.run()
        assert torch.equal(codes(self.k), want[0]) and torch.equal(codes(self.v), want[1])


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("order", ["page", "head"])
@pytest.mark.parametrize("copies", [False, True])
def test_append(kv, order, copies):
    for i, (n, hkv, d, page) in enumerate(((1, 1, 64, 1), (5, 3, 128, 8), (33, 4, 64, 64),
                                           (1, 32, 128, 16))):
        Append(n=n, hkv=hkv, d=d, page=page, pool=300 if page == 1 else 40, kv=kv, order=order,
               copies=copies, seed=i).check()


def test_append_one_layer_and_one_request():
    x = Append(layers=1, batch=1, n=2, copies=False)
    want = x.expect()
    B.paged_append(x.s, ints(x.slots), x.new[0, :, :, :3], x.new[0, :, :, 3:], x.k[0], x.v[0],
                   B.page_layout(x.k[0]))
    assert torch.equal(codes(x.k), want[0]) and torch.equal(codes(x.v), want[1])


def test_append_rounds_and_clamps():
    """Every bf16 value, NaN and infinities among them, into fp8."""
    x = Append(layers=1, batch=1, n=512, hkv=1, d=128, page=128, pool=10, kv="fp8", copies=False)
    bits = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16)
    x.new[0, 0, :, 0] = x.new[0, 0, :, 1] = bits.view(512, 128).view(torch.bfloat16)
    x.ks.fill_(1.0)
    x.vs.fill_(0.37)
    x.slots = [[(37 * i) % 1280 for i in range(512)]]
    x.run()
    new = x.new[0, 0, :, 0].float()
    at = torch.tensor(x.slots[0], device=DEV)
    for t, s in ((x.k, 1.0), (x.v, x.vs.item())):
        got = t[0, :, 0].reshape(-1, 128).view(torch.uint8)[at]
        want = e4m3(new, torch.full_like(new, s)).view(torch.uint8)
        nan = new.isnan()
        assert torch.equal(got[~nan], want[~nan]) and ((got[nan] & 127) == 127).all()


def test_copies_outside_the_pool_copy_nothing():
    x = Append(copies=True)
    x.copies.copy_(ints([[-1, 3, 4], [40, 3, 4], [2, 1 << 30, 4]]))
    x.slots = [[-1] * 5] * 3
    before = [codes(t).clone() for t in (x.k, x.v)]
    x.run()
    assert torch.equal(codes(x.k), before[0]) and torch.equal(codes(x.v), before[1])
    x.copies.copy_(ints([[5, 6, -2], [7, 7, 4], [8, 9, 1000]]))  # rows are clamped to the page
    x.run()
    before[0][:, 9], before[1][:, 9] = before[0][:, 8].clone(), before[1][:, 8].clone()
    assert torch.equal(codes(x.k), before[0]) and torch.equal(codes(x.v), before[1])


def test_append_past_two_gib():
    pool = 20000
    k = torch.zeros((pool, 4, 128, 128), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    new = torch.randn((2, 3, 8, 128), device=DEV).bfloat16()
    slots = ints([[pool * 128 - 1, 7, -1], [pool * 127, 128 * 10000 + 5, 0]])
    B.paged_append(B.make_shape(2, 4, 4, 128), slots, new[:, :, :4], new[:, :, 4:], k, v,
                   B.page_layout(k), ints([[19000, 19990, 3], [-1, -1, -1]]))
    for b in range(2):
        for i, x in enumerate(slots[b].tolist()):
            if x >= 0:
                assert torch.equal(k[x // 128, :, x % 128], new[b, i, :4])
                assert torch.equal(v[x // 128, :, x % 128], new[b, i, 4:])
    assert (k != 0).any(-1).sum() == 5 * 4


def test_captured_append():
    x = Append(kv="fp8")
    slots = ints(x.slots)
    layout = B.page_layout(x.k[0], x.ks, x.vs)
    start = [codes(t).clone() for t in (x.k, x.v)]
    want = x.expect()
    g = torch.cuda.CUDAGraph()
    args = (x.s, slots, x.new[:, :, :, :3], x.new[:, :, :, 3:], x.k, x.v, layout, x.copies)
    B.paged_append(*args)
    with torch.cuda.graph(g):
        B.paged_append(*args)
    for _ in range(3):
        codes(x.k).copy_(start[0])
        codes(x.v).copy_(start[1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(codes(x.k), want[0]) and torch.equal(codes(x.v), want[1])
