"""A KV cache in pages: the calls whose speed is measured.

A case is one pass through one operator, on inputs that already sit in GPU
memory:

* ``pages``   ``page_update`` for one step of a serving loop: requests that
              leave, requests that come with a prompt, requests that go on by
              a token; with ``beams`` above 1 after a ``page_reorder`` that
              lets beams go on from others' pages;
* ``append``  ``paged_append``: new K/V rows of the layers into their slots, and
              the rows of pages that stopped being shared;
* ``attend``  ``paged_attention`` of each layer for one token per request:
              dense, window, or diagonal (the kept rows of a plan, and the
              window logits that the selection reads);
* ``beam``    ``beam_select`` over beams and vocabulary, then ``page_reorder``.

``launch`` says how a program issues it: ``graph`` replays a HIP graph
captured on the first pass (a serving loop), ``eager`` calls the binding.

The definitions.  Row ``r`` of request ``b`` (prompt rows first, then decode
position ``j`` in row ``prompt[b] + j``) lives in page ``table[b, r // P]`` at row
``r % P``.

``page_update``: a request of length below 0 gives back all its pages, another one
those whose rows all lie between its sinks and the window of position ``length``.
Rows ``length .. length + new - 1`` get pages: an entry without one, and one whose
page has other users, takes the next free page (no user) from the cursor on, around
the pool, requests and entries in order; a request whose pages, added to those of
the requests before it, are more than there are gets none.  ``slot[b, i]`` is the
place of row ``length + i``; ``copies[b]`` the page, the new page and the rows where
the first entry was shared; ``pos[b]`` the decode position of the last row.

``paged_attention``: softmax over the rows that the mode keeps, without those whose
entry names no page.

``beam_select``: the ``beams`` best of ``score[b, w] + log_softmax(logits[b, w])[v]``,
ties to the lowest ``w * vocab + v``.
"""

from __future__ import annotations

import math

import torch

own = False

FP8_MAX = 448.0


# ---- cases -----------------------------------------------------------------------

def _named(c, name):
    return c if name is None else {**c, "name": name}


def _model(layers, batch, heads, dim, prompt, grid, page, more):
    c = {"layers": layers, "batch": batch, "q_heads": heads[0], "kv_heads": heads[1], "dim": dim,
         "prompt": prompt, "grid_h": grid[0], "grid_w": grid[1], "page": page, "mode": "dense",
         "window": 1, "n_att": 1, "sinks": 0, "kv": "bf16", "ragged": False}
    c.update(more)
    return c


def _pages(name, launch, batch, prompt, grid, page, **more):
    c = _model(1, batch, (1, 1), 64, prompt, grid, page, more)
    return _named({"op": "pages", "launch": launch, "beams": 1, **c}, name)


def _append(name, launch, layers, batch, kv_heads, dim, prompt, grid, page, **more):
    c = _model(layers, batch, (kv_heads, kv_heads), dim, prompt, grid, page, more)
    return _named({"op": "append", "launch": launch, "new": "token", "copies": False, **c}, name)


def _attend(name, launch, layers, batch, heads, dim, prompt, grid, page, **more):
    c = _model(layers, batch, heads, dim, prompt, grid, page, more)
    return _named({"op": "attend", "launch": launch, "out": "bf16", **c}, name)


def _beam(name, launch, batch, beams, vocab, logits, prompt, grid, page):
    return _named({"op": "beam", "launch": launch, "batch": batch, "beams": beams, "vocab": vocab,
                   "logits": logits, "prompt": prompt, "grid_h": grid[0], "grid_w": grid[1],
                   "page": page}, name)


def listed():
    return [
        # One LlamaGen-XL-like request being decoded: what a single step's
        # bookkeeping costs.
        _pages("pages_b1", "eager", 1, 120, (24, 24), 16),
        # Continuous batching of Janus-Pro-7B-like requests: some leave, as
        # many come with prompts of their own lengths, the others go on.
        _pages("pages_serve_b128", "graph", 128, 256, (24, 24), 16, ragged=True),
        # One token of one request into one layer: the smallest append.
        _append("append_b1", "eager", 1, 1, 20, 64, 120, (24, 24), 16),
        # Beams of a step, all 30 layers at once, half of them with a page
        # that has to be copied first.
        _append("append_beams_b32", "graph", 30, 32, 32, 128, 256, (24, 24), 16, copies=True),
        # Prompts of their own lengths into fp8 pages.
        _append("append_prompt_fp8_b32", "eager", 8, 32, 8, 128, 256, (64, 64), 64, kv="fp8",
                new="prompt", ragged=True),
        # One layer of one LlamaGen-XL-like request: the smallest attention.
        _attend("attend_b1", "eager", 1, 1, (20, 20), 64, 120, (24, 24), 16),
        # A serving batch of Janus-Pro-7B-like requests, dense: the most bytes.
        _attend("attend_janus_b128", "graph", 4, 128, (32, 32), 128, 256, (24, 24), 16,
                ragged=True),
        # Emu3-8B-like grouped heads over fp8 pages, fp32 outputs as a decode
        # step gives them.
        _attend("attend_emu3_fp8_b32", "graph", 4, 32, (32, 8), 128, 256, (64, 64), 64, kv="fp8",
                out="fp32"),
        # Algorithm 1's kept rows at 95 % sparsity, gathered from pages, with the
        # window logits that its selection reads.
        _attend("attend_diagonal_janus_b64", "graph", 4, 64, (32, 32), 128, 256, (24, 24), 16,
                mode="diagonal", window=288, n_att=29, out="fp32"),
        # StreamingLLM rows with eight query heads per KV head; pages behind
        # the window are gone; an odd grid.
        _attend("attend_window_gqa8_b24", "eager", 1, 24, (32, 4), 128, 77, (45, 61), 32,
                mode="window", n_att=1028, sinks=4, ragged=True),
        # One request's beams over an image tokenizer's 16384 codes.
        _beam("beam_b1", "eager", 1, 4, 16384, "fp32", 256, (24, 24), 16),
        # A serving batch of beams over text and image tokens, an odd number.
        _beam("beam_b32", "graph", 32, 8, 65539, "bf16", 256, (24, 24), 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    op = rng.choice(["pages", "append", "attend", "attend", "attend", "beam"])
    launch = rng.choice(["eager", "graph"])
    prompt = _log_int(rng, 16, 512)
    grid = (_log_int(rng, 12, 64), _log_int(rng, 12, 64))
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "beam":
        return _beam(None, launch, _log_int(rng, 1, 32), rng.choice([1, 2, 3, 4, 5, 8]),
                     _log_int(rng, 500, 131072), rng.choice(["fp32", "bf16"]), prompt, grid, page)
    mode = rng.choice(["dense", "window", "diagonal"])
    length = grid[0] * grid[1]
    sinks = 0 if mode == "dense" else rng.choice([0, 4])
    more = {"mode": mode, "sinks": sinks, "kv": rng.choice(["bf16", "bf16", "fp8"]),
            "ragged": rng.random() < 0.5}
    if mode == "window":
        more["n_att"] = sinks + _log_int(rng, 16, 1024)
    elif mode == "diagonal":
        more["window"] = max(sinks + 2, length // rng.choice([2, 2, 4]))
        more["n_att"] = max(sinks + 1, min(more["window"], length // rng.choice([5, 10, 20])))
    dim = rng.choice([64, 128])
    if op == "pages":
        c = _pages(None, launch, _log_int(rng, 1, 256), prompt, grid, page,
                   beams=rng.choice([1, 1, 2, 4]), **more)
        c["batch"] = max(c["beams"], c["batch"] // c["beams"] * c["beams"])
        return c
    batch = _log_int(rng, 1, 64)
    if op == "append":
        new = rng.choice(["token", "token", "prompt"])
        c = _append(None, launch, _log_int(rng, 1, 32), batch, rng.choice([4, 8, 20, 32]), dim,
                    prompt, grid, page, new=new, copies=new == "token" and rng.random() < 0.5,
                    **more)
    else:
        q_heads = rng.choice([8, 16, 20, 32, 32, 64])
        kv_heads = q_heads // rng.choice([g for g in (1, 1, 2, 4, 8) if q_heads % g == 0])
        c = _attend(None, launch, 4 if launch == "graph" else 1, batch, (q_heads, kv_heads), dim,
                    prompt, grid, page, out=rng.choice(["bf16", "fp32"]), **more)
    while c["batch"] > 1 and (any(work(c)[k] > most[k] for k in most) or _held(c) > 3e9):
        c["batch"] = max(1, c["batch"] * 3 // 4)
    return c


# ---- sizes -----------------------------------------------------------------------

def _length(c):
    return c["grid_h"] * c["grid_w"]


def _elem(c):
    return 1 if c["kv"] == "fp8" else 2


def _window(c):
    """Positions after the sinks that a step looks back on, itself included (0: all)."""
    return {"dense": 0, "window": c["n_att"] - c["sinks"], "diagonal": c["window"]}[c["mode"]]


def _prompts(c):
    """Prompt rows of each request: all, or evenly from a half to all of them."""
    n, b = c["prompt"], c["batch"]
    return [n - (n * i) // (2 * b) if c["ragged"] else n for i in range(b)]


def _positions(c):
    """Decode positions evenly over the image."""
    return [int((i + 0.5) * _length(c) / c["batch"]) for i in range(c["batch"])]


def _most_pages(c):
    """Entries of a table's row."""
    return (c["prompt"] + _length(c) + c["page"] - 1) // c["page"]


def _kept(c, t):
    """Decode rows that a step at position ``t`` attends."""
    return t + 1 if c["mode"] == "dense" else min(t + 1, c["n_att"])


def _held(c):
    """Values of the caches, or of one layer's gathered rows in fp32."""
    rows = c["kv_heads"] * c["dim"] * c["batch"]
    cache = c["layers"] * rows * (c["prompt"] + _length(c) + c["page"])
    return max(cache, 4.0 * rows * (c["prompt"] + _kept(c, _length(c))))


def _new(c):
    return c["prompt"] if c["op"] == "pages" or c["new"] == "prompt" else 1


def work(c):
    b = c["batch"]
    if c["op"] == "beam":
        size = 4 if c["logits"] == "fp32" else 2
        slots = b * c["beams"]
        pages = (c["prompt"] + _length(c) // 2) // c["page"] + 1
        return {"bytes": slots * (c["vocab"] * size + 16 + 16 * pages),
                "flops": 3 * slots * c["vocab"]}
    if c["op"] == "pages":
        # lengths and counts in; slots, positions, copies and flags out; entries
        table = 4 * (_most_pages(c) * 4 if c["beams"] > 1 else 2)
        return {"bytes": b * (8 + 4 * c["prompt"] + 20 + table), "flops": 0}
    row = 2 * c["kv_heads"] * c["dim"]  # values of a token's K and V
    if c["op"] == "append":
        rows = sum(_prompts(c)) if c["new"] == "prompt" else b
        copied = sum(n for _, n in _copied(c))
        return {"bytes": c["layers"] * row * (rows * (2 + _elem(c)) + copied * 2 * _elem(c)),
                "flops": 0}
    rows = sum(n + _kept(c, t) for n, t in zip(_prompts(c), _positions(c)))
    q = b * c["q_heads"] * c["dim"] * (2 + (4 if c["out"] == "fp32" else 2))
    logits = 0
    if c["mode"] == "diagonal":
        kept = sum(_kept(c, t) for t in _positions(c))
        logits = 4 * kept * (c["q_heads"] + c["kv_heads"])  # written, and their places read
    return {"bytes": c["layers"] * (rows * row * _elem(c) + q + logits),
            "flops": c["layers"] * 4 * c["dim"] * c["q_heads"] * rows}


# ---- inputs ----------------------------------------------------------------------

def _gen(seed, *what):
    s = seed
    for w in what:
        s = s * 1000003 + w
    return torch.Generator(device="cuda").manual_seed(s % (1 << 62))


def _randn(shape, seed, *what):
    return torch.randn(shape, generator=_gen(seed, *what), device="cuda", dtype=torch.bfloat16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _perm(n, seed, *what):
    return torch.randperm(n, generator=_gen(seed, *what), device="cuda")


def _live(c, prompt, rows):
    """``[B, M]``: the table's entries of a request of so many rows that are not
    behind its window."""
    i = torch.arange(_most_pages(c), device="cuda")
    rows = rows[:, None]
    live = i < (rows + c["page"] - 1) // c["page"]
    if c["mode"] != "dense":
        first = (prompt[:, None] + c["sinks"] + c["page"] - 1) // c["page"]
        last = torch.div(rows - _window(c), c["page"], rounding_mode="floor")
        live &= ~((i >= first) & (i < last))
    return live


def _table(seed, live, spare, pool=0):
    """Pages all over the pool for the entries in use, and how many users each has."""
    n = int(live.sum())
    pool = pool or n + spare
    table = torch.full(live.shape, -1, dtype=torch.int32, device="cuda")
    pages = _perm(pool, seed, 80)[:n].int()
    table[live] = pages
    refs = torch.zeros(pool, dtype=torch.int32, device="cuda")
    refs[pages.long()] = 1
    return table, refs


def _caches(c, seed, pages):
    """K and V of every layer ``[layers, pages, Hkv, P, d]``, and fp8 scales ``[layers, Hkv]``."""
    shape = (c["layers"], pages, c["kv_heads"], c["page"], c["dim"])
    if c["kv"] == "bf16":
        return [_randn(shape, seed, 1), _randn(shape, seed, 2), None, None]
    got, scales = [], []
    for i in (1, 2):
        t = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
        s = torch.empty(shape[0], shape[2], device="cuda")
        for layer in range(c["layers"]):
            x = _randn(shape[1:], seed, i, layer).float()
            s[layer] = x.abs().amax(dim=(0, 2, 3)) / FP8_MAX
            y = (x / s[layer][:, None, None]).clamp(-FP8_MAX, FP8_MAX)
            t[layer] = y.to(torch.float8_e4m3fn)
        got.append(t)
        scales.append(s)
    return got + scales


def _copied(c):
    """Requests of an append whose first page is copied, and the rows of it."""
    if c["op"] != "append" or not c["copies"]:
        return []
    rows = [n + t for n, t in zip(_prompts(c), _positions(c))]  # before the new token
    return [(b, n % c["page"]) for b, n in enumerate(rows) if b % 2 and n % c["page"]]


class _State:
    pass


def prepare(case, seed):
    st, c = _State(), case
    st.case, st.handles, st.step = c, None, 0
    {"pages": _prepare_pages, "append": _prepare_append, "attend": _prepare_attend,
     "beam": _prepare_beam}[c["op"]](st, c, seed)
    return st


def _prepare_pages(st, c, seed):
    """A schedule of as many steps as a request lives, around and around: in one
    it leaves, in the next it comes with its prompt, then it goes on by a token
    a step.  Beams of a group come and go together."""
    b, w = c["batch"], c["beams"]
    steps = st.steps = min(_length(c), 600) + 2
    groups = b // w
    at = torch.arange(groups, device="cuda")[_perm(groups, seed, 70)].repeat_interleave(w)
    phase = (torch.arange(steps, device="cuda")[:, None] + at * steps // groups) % steps
    prompt = _ints(_prompts(c)).view(groups, w)[:, :1].expand(groups, w).reshape(-1)
    st.prompt = prompt.contiguous()
    length = torch.where(phase == 0, -1, torch.where(phase == 1, 0, prompt + phase - 2))
    new = torch.where(phase == 0, 0, torch.where(phase == 1, prompt, 1))
    held = torch.where(phase[0] == 0, prompt + steps - 2,
                       torch.where(phase[0] == 1, 0, prompt + phase[0] - 2))
    # what requests hold on average, and some pages more
    pool = b * ((c["prompt"] + steps // 2) // c["page"] + 2) + (c["prompt"] + steps) // c["page"] + 64
    st.table, st.refs = _table(seed, _live(c, prompt.long(), held.long()), 0, pool)
    st.cursor = torch.randint(0, st.refs.numel(), (1,), generator=_gen(seed, 71), device="cuda",
                              dtype=torch.int32)
    told = [length.int(), new.int()]
    if w > 1:
        pick = torch.randint(0, w, (steps, groups, w), generator=_gen(seed, 72), device="cuda")
        first = w * torch.arange(groups, device="cuda")
        told.append((pick + first[:, None]).view(steps, b).int())
    st.told = torch.stack(told, 1)  # [steps, length and new (and parent), B]
    st.slots = torch.full((b, c["prompt"]), -1, dtype=torch.int32, device="cuda")
    st.copies = torch.full((b, 3), -1, dtype=torch.int32, device="cuda")
    st.pos = torch.full((b,), -1, dtype=torch.int32, device="cuda")
    st.flags = torch.zeros(b, dtype=torch.int32, device="cuda")
    st.now = st.told[0].clone()  # a graph reads the step's lengths at one address


def _prepare_append(st, c, seed):
    b, n = c["batch"], _new(c)
    prompt = _ints(_prompts(c)).long()
    if c["new"] == "prompt":
        first, count = torch.zeros_like(prompt), prompt
    else:
        first, count = prompt + _ints(_positions(c)).long(), torch.ones_like(prompt)
    copied = _copied(c)
    live = _live(c, prompt, first + count)
    table, refs = _table(seed, live, len(copied) + 5)
    st.k, st.v, st.k_scale, st.v_scale = _caches(c, seed, refs.numel())
    st.copies = None
    if c["copies"]:
        # the new page is the request's own, the old one somewhere else in the pool
        at = torch.tensor([i for i, _ in copied], dtype=torch.int64, device="cuda")
        st.copies = torch.full((b, 3), -1, dtype=torch.int32, device="cuda")
        st.copies[at, 0] = (refs == 0).nonzero()[:len(copied), 0].int()
        st.copies[at, 1] = table[at, first[at] // c["page"]]
        st.copies[at, 2] = (first[at] % c["page"]).int()
    row = first[:, None] + torch.arange(n, device="cuda")
    page = table.long().gather(1, (row // c["page"]).clamp(max=table.shape[1] - 1))
    slot = torch.where(row < (first + count)[:, None], page * c["page"] + row % c["page"], -1)
    st.slots, st.table = slot.int().contiguous(), table
    # K and V side by side, as a projection leaves them
    st.rows = _randn((c["layers"], b, n, 2 * c["kv_heads"], c["dim"]), seed, 3)


def _prepare_attend(st, c, seed):
    b, hq, hkv, d = c["batch"], c["q_heads"], c["kv_heads"], c["dim"]
    order = _perm(b, seed, 70)
    st.prompt = _ints(_prompts(c))[order].contiguous()
    st.pos = _ints(_positions(c))[order].contiguous()
    rows = st.prompt.long() + st.pos.long() + 1
    st.table, refs = _table(seed, _live(c, st.prompt.long(), rows), 7)
    st.k, st.v, st.k_scale, st.v_scale = _caches(c, seed, refs.numel())
    st.q = _randn((c["layers"], b, hq, d), seed, 3)
    st.out = torch.zeros((c["layers"], b, hq, d), device="cuda",
                         dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16)
    st.kept = st.logits = None
    if c["mode"] == "diagonal":
        st.kept = _random_plan(c, seed, st.pos.long())
        cap = st.kept.shape[2]
        st.logits = torch.zeros((c["layers"], b, hq, cap), device="cuda")


def _random_plan(c, seed, t):
    """``[B, Hkv, cap]`` kept decode positions in order, -1 past their number: the
    sinks, the newest and random ones of the window."""
    b, h, s, w = c["batch"], c["kv_heads"], c["sinks"], c["window"]
    cap = min(c["n_att"], _length(c))
    far = 1 << 40
    d = torch.arange(w, device="cuda")
    j = t[:, None] - d  # [B, w]
    ok = j >= s
    key = torch.rand((b, h, w), generator=_gen(seed, 73), device="cuda") + (~ok[:, None]) * 2.0
    key[:, :, 0] = torch.where(ok[:, 0], -1.0, 3.0)[:, None]
    best = key.argsort(-1)[:, :, :cap - s]
    got = j[:, None].expand(b, h, w).gather(2, best)
    got = torch.where(ok[:, None].expand(b, h, w).gather(2, best), got, far).sort(-1).values
    sink = torch.arange(s, device="cuda")
    sink = torch.where(sink <= t[:, None], sink, far)[:, None].expand(b, h, s)
    got = torch.cat([sink, got], 2).sort(-1).values
    return torch.where(got < far, got, -1).int()


def _prepare_beam(st, c, seed):
    b, w, v = c["batch"], c["beams"], c["vocab"]
    st.x = 3 * torch.randn((b, w, v), generator=_gen(seed, 1), device="cuda")
    if c["logits"] == "bf16":
        st.x = st.x.bfloat16()
    st.score = -20 * torch.rand((b, w), generator=_gen(seed, 2), device="cuda")
    rows = torch.full((b * w,), c["prompt"] + _length(c) // 2, device="cuda")
    m = {**c, "mode": "dense"}
    st.table, st.refs = _table(seed, _live(m, None, rows), 9)
    st.new_score = torch.zeros((b, w), device="cuda")
    st.parent = torch.zeros((b, w), dtype=torch.int32, device="cuda")
    st.token = torch.zeros((b, w), dtype=torch.int32, device="cuda")


# ---- the framework's calls ---------------------------------------------------------

def _handles(st):
    """What a program keeps with its buffers."""
    from paper_2609_19702_amd import binding as B
    c, h = st.case, {"graph": None}
    if c["op"] == "beam":
        h["pages"] = B.make_pages(c["page"], st.table, st.refs)
        n = B.beam_workspace_bytes(c["batch"], c["beams"], c["vocab"])
        h["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        return h
    mode = {"dense": B.MODE_DENSE, "window": B.MODE_WINDOW, "diagonal": B.MODE_DIAGONAL}[c["mode"]]
    h["p"] = B.make_params(c["prompt"], c["grid_h"], c["grid_w"], c["window"], c["n_att"], mode,
                           c["sinks"])
    h["s"] = B.make_shape(c["batch"], c["q_heads"], c["kv_heads"], c["dim"])
    if c["op"] == "pages":
        h["pages"] = B.make_pages(c["page"], st.table, st.refs, st.cursor, st.prompt)
        return h
    if c["op"] == "append":
        h["layout"] = B.page_layout(st.k[0], st.k_scale, st.v_scale)  # scales of all layers
        return h
    h["pages"] = B.make_pages(c["page"], st.table, prompt=st.prompt)
    h["scale"] = 1 / math.sqrt(c["dim"])
    scales = [(None, None) if st.k_scale is None else (st.k_scale[i], st.v_scale[i])
              for i in range(c["layers"])]
    h["layouts"] = [B.page_layout(st.k[i], *scales[i]) for i in range(c["layers"])]
    h["plan"] = None
    if st.kept is not None:
        h["plan"] = torch.zeros(B.plan_bytes(h["p"], h["s"]), dtype=torch.uint8, device="cuda")
        count, _, places = B.plan_views(h["p"], h["s"], h["plan"])
        count.copy_((st.kept >= 0).sum(2).view(-1))
        places.copy_(st.kept.clamp(min=0).view(places.shape))
    n = B.paged_workspace_bytes(h["p"], h["s"])
    h["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return h


def _issue(st):
    from paper_2609_19702_amd import binding as B
    c, h = st.case, st.handles
    if c["op"] == "pages":
        if c["beams"] > 1:
            B.page_reorder(h["pages"], st.now[2])
        B.page_update(h["p"], h["pages"], st.now[0], st.now[1], st.slots, st.pos, st.copies, st.flags)
    elif c["op"] == "append":
        hkv = c["kv_heads"]
        B.paged_append(h["s"], st.slots, st.rows[:, :, :, :hkv], st.rows[:, :, :, hkv:], st.k,
                       st.v, h["layout"], st.copies)
    elif c["op"] == "attend":
        for i in range(c["layers"]):
            B.paged_attention(h["p"], h["s"], h["pages"], st.q[i], st.k[i], st.v[i],
                              h["layouts"][i], st.pos, h["scale"], st.out[i], h["plan"],
                              None if st.logits is None else st.logits[i], h["ws"])
    else:
        B.beam_select(st.x, st.score, st.new_score, st.parent, st.token, h["ws"])
        B.page_reorder(h["pages"], st.parent.view(-1))


def _capture(st):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = {k: x.clone() for k, x in vars(st).items()
            if isinstance(x, torch.Tensor) and k in ("table", "refs", "cursor")}
    with torch.cuda.stream(side):
        _issue(st)  # loads the kernels
        for k, x in kept.items():
            getattr(st, k).copy_(x)
    torch.cuda.current_stream().wait_stream(side)
    st.handles["graph"] = torch.cuda.CUDAGraph()
    with torch.cuda.graph(st.handles["graph"]):
        _issue(st)


def _own_pass(st):
    """One pass; the first makes the handles that a program keeps with its
    buffers, and the graph where it replays one."""
    if st.handles is None:
        st.handles = _handles(st)
        if st.case["launch"] == "graph":
            _capture(st)
    if st.handles["graph"] is not None:
        st.handles["graph"].replay()
    else:
        _issue(st)


# ---- the plain forms ----------------------------------------------------------------

def _plain_reorder(table, refs, parent):
    """Every row of the table becomes its parent's (none below 0), in place."""
    at = parent.long()
    new = torch.where((at >= 0)[:, None], table[at.clamp(min=0)], -1)
    for t, sign in ((new, 1), (table, -1)):
        t = t.view(-1).long()
        refs.index_add_(0, t.clamp(min=0), ((t >= 0) * sign).int())
    table.copy_(new)


def _plain_pages(st):
    c, page = st.case, st.case["page"]
    if c["beams"] > 1:
        _plain_reorder(st.table, st.refs, st.now[2])
    length, new, prompt = st.now[0].long(), st.now[1].long(), st.prompt.long()
    pool = st.refs.numel()
    entry = torch.arange(st.table.shape[1], device="cuda")
    table = st.table.long()
    # what leaves
    gone = (length < 0)[:, None].expand(table.shape)
    if c["mode"] != "dense":
        lo = (prompt + c["sinks"] + page - 1) // page
        hi = torch.div(length - _window(c) + 1, page, rounding_mode="floor")
        gone = gone | ((entry >= lo[:, None]) & (entry < hi[:, None]))
    gone = gone & (table >= 0)
    refs = st.refs.long().index_add_(0, table.clamp(min=0).view(-1), -gone.view(-1).long())
    table = torch.where(gone, -1, table)
    # what is needed
    here = length >= 0
    end = length + new
    write = (entry >= (length // page)[:, None]) & (entry < ((end + page - 1) // page)[:, None])
    write = write & (here & (new > 0))[:, None]
    shared = write & (table >= 0) & (refs[table.clamp(min=0)] > 1)
    want = (write & (table < 0)) | shared
    need = want.sum(1)
    free = refs == 0
    ids = torch.arange(pool, device="cuda")
    order = torch.where(free, (ids - st.cursor.long()) % pool, pool + ids).argsort()
    ok = here & (end <= table.shape[1] * page)
    ok = ok & ((need == 0) | (need.cumsum(0) <= free.sum()))
    want, shared = want & ok[:, None], shared & ok[:, None]
    rank = want.view(-1).cumsum(0).view(want.shape) - 1
    old, table = table, torch.where(want, order[rank.clamp(min=0, max=pool - 1)], table)
    refs.index_add_(0, old.clamp(min=0).view(-1), -shared.view(-1).long())
    refs.index_add_(0, table.clamp(min=0).view(-1), want.view(-1).long())
    last = torch.where(want, rank, -1).amax()
    st.cursor.copy_(torch.where(last >= 0, (order[last.clamp(min=0)] + 1) % pool, st.cursor[0]))
    # what comes out
    first = (length // page).clamp(min=0, max=table.shape[1] - 1)[:, None]
    copy = shared.gather(1, first) & (length % page > 0)[:, None]
    told = torch.cat([old.gather(1, first), table.gather(1, first), (length % page)[:, None]], 1)
    st.copies.copy_(torch.where(copy, told, -1))
    i = torch.arange(st.slots.shape[1], device="cuda")
    row = length.clamp(min=0)[:, None] + i
    slot = table.gather(1, (row // page).clamp(max=table.shape[1] - 1)) * page + row % page
    st.slots.copy_(torch.where((i < new[:, None]) & ok[:, None], slot, -1))
    st.pos.copy_(torch.where(ok, end - 1 - prompt, -1).clamp(min=-1))
    st.flags.copy_(here & ~ok)
    st.table.copy_(table)
    st.refs.copy_(refs)


def _set_rows(t, page, off, x):
    """Rows ``[layers, n, Hkv, d]`` in fp32 into pages (fp8 by its bytes)."""
    x = x.to(t.dtype)
    if t.dtype is torch.float8_e4m3fn:
        t, x = t.view(torch.uint8), x.view(torch.uint8)
    t[:, page, :, off] = x.transpose(0, 1)


def _plain_append(st):
    c, hkv = st.case, st.case["kv_heads"]
    if st.copies is not None:
        src, dst, rows = st.copies.long().unbind(1)
        b, i = (torch.arange(c["page"], device="cuda") < rows[:, None]).nonzero(as_tuple=True)
        for t in (st.k, st.v):
            t = t.view(torch.uint8) if t.dtype is torch.float8_e4m3fn else t
            t[:, dst[b], :, i] = t[:, src[b], :, i]
    b, i = (st.slots >= 0).nonzero(as_tuple=True)
    slot = st.slots[b, i].long()
    for t, new, scale in ((st.k, st.rows[:, :, :, :hkv], st.k_scale),
                          (st.v, st.rows[:, :, :, hkv:], st.v_scale)):
        x = new[:, b, i].float()  # [layers, rows, Hkv, d]
        if scale is not None:
            x = (x / scale[:, None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        _set_rows(t, slot // c["page"], slot % c["page"], x)


def _attended(st):
    """``[B, 1 or Hkv, N]``: rows that a step attends, and which of them there are."""
    c = st.case
    t, prompt = st.pos.long()[:, None], st.prompt.long()[:, None]
    front = torch.arange(c["prompt"], device="cuda")
    if c["mode"] == "diagonal":
        kept = st.kept.long()
        row = torch.cat([front.expand(*kept.shape[:2], -1), prompt[:, :, None] + kept], 2)
        ok = torch.cat([(front < prompt)[:, None].expand(*kept.shape[:2], -1), kept >= 0], 2)
        return row, ok
    j = torch.arange(min(_length(c), max(_positions(c)) + 1), device="cuda").expand(c["batch"], -1)
    if c["mode"] == "window":
        s, w = c["sinks"], _window(c)
        i = torch.arange(min(c["n_att"], j.shape[1]), device="cuda")
        j = torch.where(i < s, i, torch.maximum(t - w + 1, torch.full_like(t, s)) + i - s)
    row = torch.cat([front.expand(c["batch"], -1), prompt + j], 1)
    ok = torch.cat([front < prompt, j <= t], 1)
    return row[:, None], ok[:, None]


def _gathered(t, page, off):
    """Rows ``[B, Hkv, N, d]`` of a layer's pages, in the cache's type."""
    head = torch.arange(t.shape[1], device="cuda")[None, :, None]
    if t.dtype is torch.float8_e4m3fn:
        return t.view(torch.uint8)[page, head, off].view(t.dtype)
    return t[page, head, off]


def _plain_attend(st):
    c = st.case
    b, hq, hkv, d = c["batch"], c["q_heads"], c["kv_heads"], c["dim"]
    row, ok = _attended(st)
    entry = (row // c["page"]).clamp(min=0, max=st.table.shape[1] - 1)
    page = st.table.long()[torch.arange(b, device="cuda")[:, None, None], entry]
    ok = (ok & (page >= 0))[:, :, None]
    page, off = page.clamp(min=0), row % c["page"]
    for i in range(c["layers"]):
        q = st.q[i].float().view(b, hkv, hq // hkv, d)
        k, v = _gathered(st.k[i], page, off).float(), _gathered(st.v[i], page, off).float()
        if st.k_scale is not None:
            k = k * st.k_scale[i][:, None, None]
            v = v * st.v_scale[i][:, None, None]
        z = (q @ k.transpose(2, 3)) * (1 / math.sqrt(d))
        if st.logits is not None:
            x = z[..., c["prompt"]:].reshape(b, hq, -1)
            there = (st.kept >= 0).repeat_interleave(hq // hkv, 1)
            st.logits[i] = torch.where(there, x, st.logits[i])
        z = z.masked_fill(~ok, -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True))
        z = z / z.sum(-1, keepdim=True)
        st.out[i] = (z @ v).view(b, hq, d).to(st.out.dtype)


def _plain_beam(st):
    """In 64 bits: the choice is compared as whole numbers."""
    b, w, v = st.x.shape
    x = st.x.double()
    top = x.amax(-1, keepdim=True)
    x = x - (top + torch.exp(x - top).sum(-1, keepdim=True).log()) + st.score.double()[..., None]
    best = torch.sort(x.view(b, -1), dim=-1, descending=True, stable=True)
    at = best.indices[:, :w]
    st.new_score.copy_(best.values[:, :w])
    st.parent.copy_(at // v + w * torch.arange(b, device="cuda")[:, None])
    st.token.copy_(at % v)
    _plain_reorder(st.table, st.refs, st.parent.view(-1))


def run(state):
    c = state.case
    if c["op"] == "pages":
        if c["launch"] == "graph":
            state.now.copy_(state.told[state.step])
        else:
            state.now = state.told[state.step]
        state.step = (state.step + 1) % state.steps
    if own:
        _own_pass(state)
    else:
        {"pages": _plain_pages, "append": _plain_append, "attend": _plain_attend,
         "beam": _plain_beam}[c["op"]](state)
    if c["op"] == "pages":
        return {"table": state.table, "refs": state.refs, "cursor": state.cursor,
                "slots": state.slots, "pos": state.pos, "copies": state.copies,
                "flags": state.flags}
    if c["op"] == "append":
        return {"k": state.k, "v": state.v}
    if c["op"] == "attend":
        return {"out": state.out, **({} if state.logits is None else {"logits": state.logits})}
    return {"score": state.new_score, "parent": state.parent, "token": state.token,
            "table": state.table, "refs": state.refs}


# ---- the same in 64 bits, request by request --------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None  # whole numbers
    st = prepare(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "beam": _exact_beam}[c["op"]](c, st)


def _exact_append(c, st):
    hkv, p = c["kv_heads"], c["page"]
    got = []
    for t, new, scale in ((st.k, st.rows[:, :, :, :hkv], st.k_scale),
                          (st.v, st.rows[:, :, :, hkv:], st.v_scale)):
        x = t.float().double()
        if st.copies is not None:
            for src, dst, rows in st.copies.tolist():
                if rows > 0:
                    x[:, dst, :, :rows] = x[:, src, :, :rows].clone()
        for b, row in enumerate(st.slots.tolist()):
            at = [(i, s) for i, s in enumerate(row) if s >= 0]
            y = new[:, b, [i for i, _ in at]].double()
            if scale is not None:
                y = (y / scale.double()[:, None, :, None]).clamp(-FP8_MAX, FP8_MAX)
            for n, (_, s) in enumerate(at):
                x[:, s // p, :, s % p] = y[:, n]
        got.append(x)
    return {"k": got[0], "v": got[1]}


def _exact_attend(c, st):
    hq, hkv, d, p, s = c["q_heads"], c["kv_heads"], c["dim"], c["page"], c["sinks"]
    g = hq // hkv
    out = st.out.double()
    logits = None if st.logits is None else st.logits.double()
    for b, (t, front) in enumerate(zip(st.pos.tolist(), st.prompt.tolist())):
        entries = st.table[b].tolist()
        if c["mode"] == "diagonal":
            kept = [[j for j in line if j >= 0] for line in st.kept[b].tolist()]
        else:
            kept = [[j for j in range(t + 1)
                     if c["mode"] == "dense" or j < s or t - j < _window(c)]] * hkv
        rows = [list(range(front)) + [front + j for j in line] for line in kept]
        there = [[r for r in line if entries[r // p] >= 0] for line in rows]
        assert there == rows  # what a step attends has a page
        place = torch.tensor([[entries[r // p] * p + r % p for r in line] for line in rows],
                             device="cuda")  # [Hkv, N]
        for i in range(c["layers"]):
            head = torch.arange(hkv, device="cuda")[:, None]
            k, v = (x[i].view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x[i]
                    for x in (st.k, st.v))
            k, v = (x[place // p, head, place % p] for x in (k, v))
            if st.k_scale is not None:
                k, v = (x.view(torch.float8_e4m3fn).float() for x in (k, v))
                k = k.double() * st.k_scale[i].double()[:, None, None]
                v = v.double() * st.v_scale[i].double()[:, None, None]
            z = st.q[i, b].double().view(hkv, g, d) @ k.double().transpose(1, 2).contiguous()
            z = z / math.sqrt(d)
            if logits is not None:
                logits[i, b, :, :len(kept[0])] = z[:, :, front:].reshape(hq, -1)
            out[i, b] = (torch.softmax(z, -1) @ v.double()).view(hq, d)
    return {"out": out, **({} if logits is None else {"logits": logits})}


def _exact_beam(c, st):
    score = torch.empty(st.score.shape, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        x = torch.log_softmax(st.x[b].double(), -1) + st.score[b].double()[:, None]
        score[b] = x.view(-1).topk(c["beams"]).values
    return {"score": score, "parent": None, "token": None, "table": None, "refs": None}
