"""Several tokens of a request at once: the calls whose speed is measured.

A case is one pass through one operator, on inputs that already sit in GPU
memory:

* ``tree``    ``tree_plan``, then ``tree_attention`` of each layer, for a tree
              of drafted tokens per request over the KV cache;
* ``chunk``   ``tree_attention`` of a chain: the next tokens of a prompt or of
              an image, all known, over what the cache holds before them;
* ``verify``  ``tree_verify``: which drafted tokens the target's probabilities
              accept, and the token that follows;
* ``append``  ``kv_append``: the K/V rows of accepted (or known) tokens into
              the caches of every layer.

``launch`` says how a program issues it: ``graph`` replays a HIP graph
captured on the first pass (a serving loop), ``eager`` calls the binding.

The definition.  Node ``i`` of request ``b`` stands at decode position ``p =
base[b] + depth(i)`` (in a chain its depth is ``i``); position ``j < 0`` is
prompt row ``prompt + j``.  It attends a cached position ``j < base[b]`` where
``j < sinks`` or ``p - j < W``, and the node ``m`` where ``m`` is ``i`` or an
ancestor of ``i`` and the same holds for ``m``'s position; ``W = n_att -
sinks`` in window mode, no bound (and no sinks) in dense mode.
"""

from __future__ import annotations

import math

import torch

own = False

FP8_MAX = 448.0


# ---- cases -----------------------------------------------------------------------

def _attention(name, op, launch, layers, batch, heads, dim, prompt, grid, nodes, start, **more):
    c = {"op": op, "launch": launch, "layers": layers, "batch": batch, "q_heads": heads[0],
         "kv_heads": heads[1], "dim": dim, "prompt": prompt, "grid_h": grid[0], "grid_w": grid[1],
         "nodes": nodes, "start": start, "mode": "dense", "n_att": 1, "sinks": 0, "ring": False,
         "kv": "bf16", "out": "bf16", "ragged": False, "branch": 3 if op == "tree" else 0}
    c.update(more)
    return _named(c, name)


def _verify(name, launch, batch, nodes, branch, vocab, draft):
    return _named({"op": "verify", "launch": launch, "batch": batch, "nodes": nodes,
                   "branch": branch, "vocab": vocab, "draft": draft}, name)


def _append(name, launch, layers, batch, kv_heads, dim, prompt, grid, nodes, start, **more):
    c = {"op": "append", "launch": launch, "layers": layers, "batch": batch, "kv_heads": kv_heads,
         "q_heads": kv_heads, "dim": dim, "prompt": prompt, "grid_h": grid[0], "grid_w": grid[1],
         "nodes": nodes, "start": start, "mode": "dense", "n_att": 1, "sinks": 0, "ring": False,
         "kv": "bf16", "path": True, "branch": 3}
    c.update(more)
    return _named(c, name)


def _named(c, name):
    return c if name is None else {**c, "name": name}


def listed():
    return [
        # One layer of the smallest speculation: one request, a few drafts.
        # What a single call costs.
        _attention("tree_b1", "tree", "eager", 1, 1, (20, 20), 64, 120, (24, 24), 7, "spread"),
        # One Janus-Pro-7B-like image being decoded, all 30 layers of a step.
        _attention("tree_janus_b1", "tree", "graph", 30, 1, (32, 32), 128, 256, (24, 24), 16,
                   "spread"),
        # A serving batch of the same heads with fp32 outputs, as a decode
        # step gives them; requests draft differently many tokens.
        _attention("tree_janus_b32", "tree", "eager", 1, 32, (32, 32), 128, 256, (24, 24), 16,
                   "spread", out="fp32", ragged=True),
        # The Emu3-8B-like grouped-query batch over an fp8 cache.
        _attention("tree_emu3_fp8_b32", "tree", "graph", 4, 32, (32, 8), 128, 256, (64, 64), 13,
                   "spread", kv="fp8", ragged=True),
        # Large trees with eight query heads per KV head (more query rows than
        # one tile), StreamingLLM rows over a ring cache.
        _attention("tree_ring_gqa8_b24", "tree", "eager", 1, 24, (32, 4), 128, 77, (45, 61), 61,
                   "spread", mode="window", n_att=1028, sinks=4, ring=True, branch=4),
        # A batch of prompts on its way into an empty cache (classifier-free
        # guidance doubles the requests of a program).
        _attention("chunk_prompt_b16", "chunk", "eager", 1, 16, (32, 32), 128, 256, (24, 24), 256,
                   "prompt", ragged=True),
        # A whole 64 x 64 image of known tokens after its prompt, as for
        # editing an image: the most arithmetic of the list.
        _attention("chunk_image_dense", "chunk", "eager", 1, 2, (32, 8), 128, 256, (64, 64), 4096,
                   "image"),
        # Its sliding-window form with sinks, from the prompt's first token.
        _attention("chunk_image_window", "chunk", "eager", 1, 2, (32, 8), 128, 256, (64, 64), 4352,
                   "prompt", mode="window", n_att=516, sinks=4, out="fp32"),
        # One request's chain of drafts against an image tokenizer's 16384
        # codes.
        _verify("verify_chain_b1", "eager", 1, 6, 1, 16384, True),
        # Trees of a serving batch, a vocabulary of text and image tokens of
        # odd size.
        _verify("verify_tree_b64", "eager", 64, 24, 3, 65539, True),
        # The accepted rows of one request into 30 layers' caches.
        _append("append_b1", "eager", 30, 1, 32, 128, 256, (24, 24), 16, "spread"),
        # Prompts into fp8 caches: the most rows of the list.
        _append("append_prompt_fp8_b32", "eager", 4, 32, 8, 128, 256, (24, 24), 256, "prompt",
                kv="fp8", path=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    op = rng.choice(["tree", "tree", "tree", "chunk", "chunk", "verify", "append"])
    launch = rng.choice(["eager", "graph"])
    if op == "verify":
        branch = rng.choice([1, 2, 3, 4])
        c = _verify(None, launch, _log_int(rng, 1, 64), _log_int(rng, 1, 32), branch,
                    _log_int(rng, 500, 131072), rng.random() < 0.7)
    else:
        dim = rng.choice([64, 128])
        prompt = _log_int(rng, 16, 512)
        grid = (_log_int(rng, 12, 64), _log_int(rng, 12, 64))
        batch = _log_int(rng, 1, 32)
        mode = rng.choice(["dense", "window"])
        sinks = 0 if mode == "dense" else rng.choice([0, 4])
        more = {"mode": mode, "sinks": sinks, "kv": rng.choice(["bf16", "bf16", "fp8"]),
                "n_att": 1 if mode == "dense" else sinks + _log_int(rng, 16, 1024),
                "ring": mode == "window" and rng.random() < 0.4}
        layers = 4 if launch == "graph" else 1
        if op == "append":
            path = rng.random() < 0.6
            c = _append(None, launch, _log_int(rng, 1, 32), batch, rng.choice([4, 8, 20, 32]), dim,
                        prompt, grid, _log_int(rng, 1, 64) if path else _log_int(rng, 1, prompt),
                        "spread" if path else "prompt", path=path, **more)
        else:
            q_heads = rng.choice([8, 16, 20, 32, 32, 64])
            kv_heads = q_heads // rng.choice([g for g in (1, 1, 2, 4, 8) if q_heads % g == 0])
            more.update(out=rng.choice(["bf16", "bf16", "fp32"]), ragged=rng.random() < 0.5)
            start = "spread" if op == "tree" else rng.choice(["prompt", "image", "spread"])
            length = grid[0] * grid[1]
            longest = {"spread": length // 2, "image": length, "prompt": prompt + length}[start]
            nodes = _log_int(rng, 1, 64) if op == "tree" else _log_int(rng, 65, max(66, longest))
            if op == "tree":
                more.update(branch=rng.choice([1, 2, 3, 4]))
            c = _attention(None, op, launch, layers, batch, (q_heads, kv_heads), dim, prompt, grid,
                           min(nodes, longest), start, **more)
    while c["batch"] > 1 and (any(work(c)[k] > most[k] for k in most) or _held(c) > 2e9):
        c["batch"] = max(1, c["batch"] * 3 // 4)
    return c


# ---- sizes -----------------------------------------------------------------------

def _length(c):
    return c["grid_h"] * c["grid_w"]


def _elem(c):
    return 1 if c["kv"] == "fp8" else 2


def _window(c):
    """W of the definition."""
    return c["n_att"] - c["sinks"] if c["mode"] == "window" else 1 << 30


def _ring_rows(c):
    """Decode rows of a ring cache: the least that window mode allows (0: linear)."""
    return c["n_att"] if c["ring"] and c["n_att"] < _length(c) else 0


def _rows(c):
    return c["prompt"] + (_ring_rows(c) or _length(c))


def _held(c):
    """Values of the larger of a pass's arrays and of its plain form's."""
    if c["op"] == "verify":
        return 8.0 * c["batch"] * c["nodes"] * c["vocab"]
    cache = c["layers"] * c["batch"] * c["kv_heads"] * _rows(c) * c["dim"] * 2
    if c["op"] == "append":
        return cache
    keys = c["prompt"] + _length(c) + c["nodes"]
    return max(cache, 2.0 * c["batch"] * c["q_heads"] * c["nodes"] * keys)


def _bases(c):
    """Decode position of each request's first node, as the requests come:
    evenly over the image ("spread"), before the image, or before the prompt."""
    if c["start"] == "prompt":
        return [-c["prompt"]] * c["batch"]
    if c["start"] == "image":
        return [0] * c["batch"]
    room = _length(c) - c["nodes"]
    return [max(0, int((i + 0.5) * room / c["batch"])) for i in range(c["batch"])]


def _counts(c):
    """Nodes of each request: all, or evenly from a half to all of them."""
    n, b = c["nodes"], c["batch"]
    if not c.get("ragged"):
        return [n] * b
    return [max(1, n - (n * i) // (2 * b)) for i in range(b)]


def _prefix_sum(p, n):
    """Sum over q in [p, p + n) of q."""
    return n * p + n * (n - 1) // 2


def work(c):
    b = c["batch"]
    if c["op"] == "verify":
        # tokens, parents, random numbers and the drafts' own probabilities,
        # then the row that the next token is drawn from
        scalars = c["nodes"] * (4 + 4 + 4 + (8 if c["draft"] else 4))
        return {"bytes": b * (scalars + 4 * c["vocab"] * (2 if c["draft"] else 1)
                              + 4 * (c["nodes"] + 2)),
                "flops": b * c["vocab"] * (3 if c["draft"] else 1)}
    row = 2 * c["kv_heads"] * c["dim"]  # values of a token's K and V
    if c["op"] == "append":
        rows = sum(_lengths(c))
        return {"bytes": c["layers"] * rows * row * (2 + _elem(c)), "flops": 0}
    w, total, flops = _window(c), 0, 0
    for base, n in zip(_bases(c), _counts(c)):
        reach = max(0, base) - max(min(c["sinks"], max(0, base)), base - w + 1, 0)
        cached = c["prompt"] + min(0, base) + min(c["sinks"], max(0, base)) + max(0, reach)
        total += row * (cached * _elem(c) + 2 * n)
        total += n * c["q_heads"] * c["dim"] * (2 + (4 if c["out"] == "fp32" else 2))
        if c["op"] == "tree":  # a node's ancestors: few beside the cache
            pairs = n * cached + n * (1 + int(math.log2(n)) if c["branch"] > 1 else (n + 1) / 2)
        else:  # every earlier position, or the window's
            pairs = 0
            full = c["prompt"] + c["sinks"]  # positions below `sinks` are never out of reach
            for lo, hi in ((base, min(base + n, c["sinks"] + w)),
                           (max(base, c["sinks"] + w), base + n)):
                if hi > lo:
                    near = hi <= c["sinks"] + w
                    pairs += (_prefix_sum(c["prompt"] + lo + 1, hi - lo) if near
                              else (hi - lo) * (full + w))
        flops += 4 * c["dim"] * c["q_heads"] * pairs
    return {"bytes": c["layers"] * total, "flops": c["layers"] * flops}


# ---- inputs ----------------------------------------------------------------------

def _gen(seed, *what):
    s = seed
    for w in what:
        s = s * 1000003 + w
    return torch.Generator(device="cuda").manual_seed(s % (1 << 62))


def _randn(shape, seed, *what):
    return torch.randn(shape, generator=_gen(seed, *what), device="cuda", dtype=torch.bfloat16)


def _perm(c, seed):
    return torch.randperm(c["batch"], generator=_gen(seed, 90), device="cuda")


def _parents(c, seed, what=91):
    """A random tree of each request: every node hangs on an earlier one that
    has fewer than ``branch`` children, the next free place or a random one."""
    b, n, most = c["batch"], c["nodes"], c["branch"]
    pick = torch.rand((b, n), generator=_gen(seed, what), device="cuda").tolist()
    rows = []
    for r in range(b):
        row, free = [-1], [[0, most]]
        for i in range(1, n):
            k = int(pick[r][i] * len(free))
            row.append(free[k][0])
            free[k][1] -= 1
            if not free[k][1]:
                free.pop(k)
            free.append([i, most])
        rows.append(row)
    return rows


def _path_of(parents, leaf):
    at = [leaf]
    while parents[at[-1]] >= 0:
        at.append(parents[at[-1]])
    return at[::-1]


def _paths(c, seed):
    """The accepted nodes of each request of an append: a path of a random tree."""
    got = []
    for r, row in enumerate(_parents(c, seed)):
        at = _path_of(row, (r * 7 + len(row) // 2) % len(row))
        got.append(at + [-1] * (c["nodes"] - len(at)))
    return got


def _lengths(c):
    """Rows of each request that an append writes, about: for ``work``."""
    n = c["nodes"]
    if not c["path"]:
        return [min(n, c["prompt"]) if c["start"] == "prompt" else n] * c["batch"]
    return [1 + math.log2(n) if c["branch"] > 1 else n] * c["batch"]


def _caches(c, seed):
    """K and V of every layer ``[layers, B, Hkv, rows, d]``, and fp8 scales."""
    shape = (c["layers"], c["batch"], c["kv_heads"], _rows(c), c["dim"])
    if c["kv"] == "bf16":
        return [_randn(shape, seed, 1), _randn(shape, seed, 2), None, None]
    got, scales = [], []
    for i in (1, 2):
        x = _randn(shape, seed, i).float()
        s = x.abs().amax(dim=(3, 4)) / FP8_MAX
        got.append((x / s[..., None, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn))
        scales.append(s.reshape(c["layers"], -1).contiguous())
    return got + scales


def _rows_of(t, row):
    """Rows of ``[..., rows, d]`` as fp32 (indexing is not there for fp8)."""
    if t.dtype is torch.float8_e4m3fn:
        return t.view(torch.uint8).index_select(-2, row).view(t.dtype).float()
    return t.index_select(-2, row).float()


class _State:
    pass


def prepare(case, seed):
    st, c = _State(), case
    st.case, st.handles = c, None
    b, n = c["batch"], c["nodes"]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    if c["op"] == "verify":
        _prepare_verify(st, c, seed)
        return st
    perm = _perm(c, seed)
    st.base = ints(_bases(c))[perm].contiguous()
    st.k, st.v, st.k_scale, st.v_scale = _caches(c, seed)
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["dim"]
    if c["op"] == "append":
        # K and V side by side, as a projection leaves them
        st.new = _randn((c["layers"], b, n, 2 * hkv, d), seed, 3)
        st.path = st.accepted = None
        if c["path"]:
            st.path = ints(_paths(c, seed))
            st.accepted = (st.path >= 0).sum(1).to(torch.int32)
        return st
    st.qkv = _randn((c["layers"], b, n, hq + 2 * hkv, d), seed, 3)
    st.count = ints(_counts(c))[perm].contiguous() if c["ragged"] else None
    st.parent = ints(_parents(c, seed)) if c["op"] == "tree" else None
    st.out = torch.zeros((c["layers"], b, n, hq, d), device="cuda",
                         dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16)
    return st


def _prepare_verify(st, c, seed):
    """Target and draft distributions that partly agree, and drafts drawn
    from the draft's (or its most likely ones, where there is no draft row)."""
    b, n, v = c["batch"], c["nodes"], c["vocab"]
    parents = _parents(c, seed)
    st.parent = torch.tensor(parents, dtype=torch.int32, device="cuda")
    z = 3 * torch.randn((b, n, v), generator=_gen(seed, 1), device="cuda")
    st.target = torch.softmax(z, -1)
    z += torch.randn((b, n, v), generator=_gen(seed, 2), device="cuda")
    at = st.parent.clamp(min=0).long()
    if c["draft"]:
        st.draft = torch.softmax(z, -1)
        rows = st.draft.gather(1, at[..., None].expand(b, n, v)).reshape(b * n, v)
        st.tokens = torch.multinomial(rows, 1, generator=_gen(seed, 3)).view(b, n).int()
    else:
        st.draft = None
        rank = (torch.tril(st.parent[:, :, None] == st.parent[:, None, :], -1)).sum(2)
        best = z.topk(min(v, c["branch"] + 1), -1).indices
        st.tokens = best[torch.arange(b, device="cuda")[:, None], at, rank].int()
    st.uniform = torch.rand((b, n + 1), generator=_gen(seed, 4), device="cuda")
    st.path = torch.zeros((b, n), dtype=torch.int32, device="cuda")
    st.accepted = torch.zeros(b, dtype=torch.int32, device="cuda")
    st.token = torch.zeros(b, dtype=torch.int32, device="cuda")


# ---- the framework's calls ---------------------------------------------------------

def _issue(st):
    from paper_2609_19702_amd import binding as B
    c, h = st.case, st.handles
    if c["op"] == "verify":
        B.tree_plan(st.parent, None, h["plan"])
        B.tree_verify(h["tree"], st.tokens, st.target, st.draft, st.uniform, st.path, st.accepted,
                      st.token)
    elif c["op"] == "append":
        hkv = c["kv_heads"]
        B.kv_append(h["p"], h["s"], h["tree"], st.new[:, :, :, :hkv], st.new[:, :, :, hkv:], st.k,
                    st.v, h["layout"], st.path, st.accepted)
    else:
        hq, hkv = c["q_heads"], c["kv_heads"]
        if st.parent is not None:
            B.tree_plan(st.parent, st.count, h["plan"])
        for i in range(c["layers"]):
            x = st.qkv[i]
            B.tree_attention(h["p"], h["s"], h["tree"], x[:, :, :hq], x[:, :, hq:hq + hkv],
                             x[:, :, hq + hkv:], st.k[i], st.v[i], h["layouts"][i], h["scale"],
                             st.out[i], h["ws"])


def _own_pass(st):
    """One pass; the first makes the handles that a program keeps with its
    buffers, and the graph where it replays one."""
    c = st.case
    if st.handles is None:
        from paper_2609_19702_amd import binding as B
        h = st.handles = {"graph": None}
        tree = c["op"] != "append" and st.parent is not None
        h["plan"] = torch.zeros(B.tree_plan_bytes(c["batch"], c["nodes"]), dtype=torch.uint8,
                                device="cuda") if tree else None
        if c["op"] == "verify":
            h["tree"] = B.make_tree(c["nodes"], plan=h["plan"])
        else:
            h["p"] = B.make_params(c["prompt"], c["grid_h"], c["grid_w"], 1, c["n_att"],
                                   B.MODE_DENSE if c["mode"] == "dense" else B.MODE_WINDOW,
                                   c["sinks"])
            h["s"] = B.make_shape(c["batch"], c["q_heads"], c["kv_heads"], c["dim"])
            h["tree"] = B.make_tree(c["nodes"], st.base, getattr(st, "count", None), h["plan"])
            h["scale"] = 1 / math.sqrt(c["dim"])
            scales = [(None, None) if st.k_scale is None else (st.k_scale[i], st.v_scale[i])
                      for i in range(c["layers"])]
            h["layouts"] = [B.kv_layout(st.k[i], ring_rows=_ring_rows(c), k_scale=scales[i][0],
                                        v_scale=scales[i][1]) for i in range(c["layers"])]
            h["layout"] = B.kv_layout(st.k[0], ring_rows=_ring_rows(c), k_scale=st.k_scale,
                                      v_scale=st.v_scale)  # an append's, of all layers
            if c["op"] != "append":
                n = B.tree_workspace_bytes(h["p"], h["s"], c["nodes"])
                h["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        if c["launch"] == "graph":
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                _issue(st)  # loads the kernels
            torch.cuda.current_stream().wait_stream(side)
            h["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(h["graph"]):
                _issue(st)
    if st.handles["graph"] is not None:
        st.handles["graph"].replay()
    else:
        _issue(st)


# ---- the plain forms ----------------------------------------------------------------

def _ancestors(parent):
    """``[B, N, N]``: whether column m is row i or an ancestor of it."""
    n = parent.shape[1]
    step = (parent[:, :, None] == torch.arange(n, device=parent.device)).double()
    reach = torch.eye(n, device=parent.device, dtype=torch.float64) + step
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (reach @ reach).clamp(max=1)
    return reach > 0


def _plain_attention(st):
    c = st.case
    b, n, hq, hkv, d = c["batch"], c["nodes"], c["q_heads"], c["kv_heads"], c["dim"]
    idx = torch.arange(n, device="cuda")
    if st.parent is None:
        seen = (idx[None, :] <= idx[:, None]).expand(b, n, n)
        depth = idx.expand(b, n)
    else:
        seen = _ancestors(st.parent)
        depth = seen.sum(2) - 1
    base = st.base.long()
    at = base[:, None] + depth  # [B, N] decode positions
    held = min(_length(c), max(_bases(c)))  # cached positions -prompt .. held - 1 of some request
    j = torch.arange(-c["prompt"], max(held, -c["prompt"]), device="cuda")
    row = c["prompt"] + j
    ring = _ring_rows(c)
    if ring:
        s = c["sinks"]
        row = torch.where(j < s, row, c["prompt"] + s + (j - s) % (ring - s))
    reach = lambda p, x: (x < c["sinks"]) | (p - x < _window(c))  # noqa: E731
    see_old = (j < base[:, None, None]) & reach(at[:, :, None], j)  # [B, N, rows]
    see_new = seen & reach(at[:, :, None], at[:, None, :])
    see = torch.cat([see_old, see_new], 2)[:, None, :, None, :]  # [B, 1, N, 1, keys]
    for i in range(c["layers"]):
        x = st.qkv[i].float()
        q = x[:, :, :hq].view(b, n, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4)
        k, v = _rows_of(st.k[i], row), _rows_of(st.v[i], row)
        if st.k_scale is not None:
            k = k * st.k_scale[i].view(b, hkv, 1, 1)
            v = v * st.v_scale[i].view(b, hkv, 1, 1)
        k = torch.cat([k, x[:, :, hq:hq + hkv].transpose(1, 2)], 2)
        v = torch.cat([v, x[:, :, hq + hkv:].transpose(1, 2)], 2)
        z = q.reshape(b, hkv, -1, d) @ k.transpose(2, 3)
        z = (z * (1 / math.sqrt(d))).view(b, hkv, n, hq // hkv, -1)
        z = z.masked_fill(~see, -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True))
        z = z / z.sum(-1, keepdim=True)
        o = (z.view(b, hkv, n * (hq // hkv), -1) @ v).view(b, hkv, n, -1, d)
        o = o.permute(0, 2, 1, 3, 4).reshape(b, n, hq, d).to(st.out.dtype)
        if st.count is not None:  # nodes past a request's count stay as they are
            o = torch.where((idx < st.count[:, None])[..., None, None], o, st.out[i])
        st.out[i] = o


def _residual(r, z, q):
    """What a rejected draft leaves of ``r / z``, and its sum."""
    r = (r / z - q).clamp(min=0)
    return r, r.sum(-1, keepdim=True)


def _plain_verify(st):
    """Sums and comparisons in 64 bits: decisions are compared as whole numbers."""
    c = st.case
    b, n, v = c["batch"], c["nodes"], c["vocab"]
    parent, token = st.parent.long(), st.tokens.long()
    node = torch.arange(n, device="cuda")
    u, end = st.uniform[:, :n].double(), st.uniform[:, n].double()
    same = parent[:, :, None] == parent[:, None, :]
    rank = torch.tril(same, -1).sum(2)  # earlier children of the same parent
    up = parent.clamp(min=0)
    batch = torch.arange(b, device="cuda")[:, None]
    most = c["branch"]
    ok = torch.zeros((b, n), dtype=torch.bool, device="cuda")
    one = torch.ones((b, n, 1), dtype=torch.float64, device="cuda")
    if st.draft is not None:
        r, z, q = st.target.double(), one, st.draft.double()
        qx = q[batch, up, token]
        for k in range(most):
            good = u * qx * z[batch, up, 0] < r[batch, up, token]
            ok |= good & (rank == k)
            if k + 1 < most:
                r, z = _residual(r, z, q)
    else:  # each draft is certain: a rejected one leaves the row without its token
        p = st.target.double()[batch, up, token]
        earlier = torch.tril(same, -1)
        again = (earlier & (token[:, :, None] == token[:, None, :])).any(2)
        left = 1 - (earlier.double() @ (p * ~again)[..., None])[..., 0]
        ok = ~again & (u * left < p)
    ok &= parent >= 0
    first = ok & ~(torch.tril(same & ok[:, None, :], -1).any(2))
    first[:, 0] = True
    seen = _ancestors(st.parent)
    on = ~(seen & ~first[:, None, :]).any(2)  # every node above it (and it) was taken
    length = on.sum(1)
    last = torch.where(on, node, -1).amax(1)
    kids = (parent == last[:, None]).sum(1)
    rows = torch.arange(b, device="cuda")
    r = st.target[rows, last].double()
    if st.draft is not None:
        q, z = st.draft[rows, last].double(), one[:, 0]
        for k in range(most):
            s, t = _residual(r, z, q)
            more = (k < kids)[:, None] & (t > 0)
            r, z = torch.where(more, s, r), torch.where(more, t, z)
    else:
        gone = torch.zeros((b, v), dtype=torch.float64, device="cuda")
        gone.scatter_add_(1, token, (parent == last[:, None]).double())
        r = torch.where(gone > 0, 0.0, r)
    upto = r.cumsum(-1)
    st.token.copy_((upto <= end[:, None] * upto[:, -1:]).sum(-1).clamp(max=v - 1))
    st.accepted.copy_(length)
    order = torch.where(on, node, n).sort(1).values
    st.path.copy_(torch.where(order < n, order, -1))


def _plain_append(st):
    c = st.case
    n, hkv = c["nodes"], c["kv_heads"]
    i = torch.arange(n, device="cuda")
    pos = st.base.long()[:, None] + i  # [B, N]: where accepted node i goes
    keep = (i < (n if st.accepted is None else st.accepted[:, None])) & (pos < _length(c))
    keep = keep.expand(c["batch"], n)
    row = c["prompt"] + pos
    ring = _ring_rows(c)
    if ring:
        s = c["sinks"]
        end = torch.where(keep, pos, -c["prompt"] - 1).amax(1, keepdim=True)
        keep = keep & ((pos < s) | (pos + ring - s > end))  # the last of a slot's rows stays
        row = torch.where(pos < s, row, c["prompt"] + s + (pos - s) % (ring - s))
    b, i = keep.nonzero(as_tuple=True)
    node = i if st.path is None else st.path.long()[b, i]
    row = row[b, i]
    for t, new, scale in ((st.k, st.new[:, :, :, :hkv], st.k_scale),
                          (st.v, st.new[:, :, :, hkv:], st.v_scale)):
        x = new[:, b, node].float()  # [layers, rows, Hkv, d]
        if scale is not None:
            s = scale.view(c["layers"], c["batch"], hkv)[:, b]
            x = (x / s[..., None]).clamp(-FP8_MAX, FP8_MAX)
        if t.dtype is torch.float8_e4m3fn:
            t.view(torch.uint8)[:, b, :, row] = x.to(t.dtype).view(torch.uint8).transpose(0, 1)
        else:
            t[:, b, :, row] = x.to(t.dtype).transpose(0, 1)


def run(state):
    c = state.case
    if own:
        _own_pass(state)
    elif c["op"] == "verify":
        _plain_verify(state)
    elif c["op"] == "append":
        _plain_append(state)
    else:
        _plain_attention(state)
    if c["op"] == "verify":
        return {"path": state.path, "accepted": state.accepted, "token": state.token}
    if c["op"] == "append":
        return {"k": state.k, "v": state.v}
    return {"out": state.out}


# ---- the same in 64 bits, node by node ------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "verify":
        return None  # whole numbers
    st = prepare(c, seed)
    return _exact_append(c, st) if c["op"] == "append" else _exact_attention(c, st)


def _place(c, j):
    """Cache row of decode position ``j``."""
    ring = _ring_rows(c)
    if ring and j >= c["sinks"]:
        return c["prompt"] + c["sinks"] + (j - c["sinks"]) % (ring - c["sinks"])
    return c["prompt"] + j


def _exact_attention(c, st):
    hq, hkv, d, w, s = c["q_heads"], c["kv_heads"], c["dim"], _window(c), c["sinks"]
    nodes = c["nodes"]
    out = st.out.double()
    parents = st.parent.tolist() if st.parent is not None else None
    counts = st.count.tolist() if st.count is not None else [nodes] * c["batch"]
    for b, base in enumerate(st.base.tolist()):
        near = list(range(-c["prompt"], min(base, s)))  # always in reach
        first = max(s if base > s else base, base - w + 1)
        cached = near + [j for j in range(max(first, min(base, s)), base)]
        rows = torch.tensor([_place(c, j) for j in cached], dtype=torch.int64, device="cuda")
        held = torch.tensor(cached, dtype=torch.int64, device="cuda")
        for layer in range(c["layers"]):
            x = st.qkv[layer][b].double()
            k, v = (_rows_of(t[layer][b], rows).double() for t in (st.k, st.v))
            if st.k_scale is not None:
                k = k * st.k_scale[layer].view(c["batch"], hkv)[b].double()[:, None, None]
                v = v * st.v_scale[layer].view(c["batch"], hkv)[b].double()[:, None, None]
            k = torch.cat([k, x[:, hq:hq + hkv].transpose(0, 1)], 1).contiguous()
            v = torch.cat([v, x[:, hq + hkv:].transpose(0, 1)], 1).contiguous()
            for i in range(counts[b]):
                q = x[i, :hq].view(hkv, hq // hkv, d)
                if parents is None:
                    # positions and keys are consecutive but for the window's gap
                    p = base + i
                    lo = len(near) + max(0, p - w + 1 - first) if first < base else len(near)
                    lo = min(lo, len(cached))
                    a = max(0, p - w + 1 - base)
                    a0 = min(max(0, s - base), a)  # nodes at sink positions (or in the prompt)
                    parts = [(0, len(near)), (lo, len(cached)),
                             (len(cached), len(cached) + a0), (len(cached) + a, len(cached) + i + 1)]
                    kk = torch.cat([k[:, f:t] for f, t in parts], 1)
                    vv = torch.cat([v[:, f:t] for f, t in parts], 1)
                else:
                    line = _path_of(parents[b], i)
                    p = base + len(line) - 1
                    ok = (held < s) | (p - held < w)
                    mine = [len(cached) + m for e, m in enumerate(line)
                            if base + e < s or p - (base + e) < w]
                    take = torch.cat([ok.nonzero()[:, 0],
                                      torch.tensor(mine, dtype=torch.int64, device="cuda")])
                    kk, vv = k[:, take], v[:, take]
                z = (q @ kk.transpose(1, 2)) / math.sqrt(d)
                out[layer, b, i] = (torch.softmax(z, -1) @ vv).reshape(hq, d)
    return {"out": out}


def _exact_append(c, st):
    hkv = c["kv_heads"]
    got = []
    for t, new, scale in ((st.k, st.new[:, :, :, :hkv], st.k_scale),
                          (st.v, st.new[:, :, :, hkv:], st.v_scale)):
        x = t.float().double()
        for b, base in enumerate(st.base.tolist()):
            line = list(range(c["nodes"]))
            if st.path is not None:
                line = [m for m in st.path[b].tolist() if m >= 0]
            for e, m in enumerate(line):
                if base + e >= _length(c):
                    continue
                y = new[:, b, m].double()
                if scale is not None:
                    y = y / scale.view(c["layers"], c["batch"], hkv)[:, b].double()[..., None]
                    y = y.clamp(-FP8_MAX, FP8_MAX)
                x[:, b, :, _place(c, base + e)] = y
        got.append(x)
    return {"k": got[0], "v": got[1]}
