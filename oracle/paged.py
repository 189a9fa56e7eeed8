"""A KV cache in pages, and a beam search's choice: fp64 and whole-number
references, request by request.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

Row ``r`` of a request (its prompt rows, then decode position ``j`` in row
``prompt + j``) is row ``r % P`` of page ``table[r // P]``; an entry outside the pool
names no page.
"""

from __future__ import annotations

import math

import numpy as np

NO_PAGES, TOO_LONG = 1, 2


def attended_positions(mode, t, n_att, sinks, kept=None):
    """Decode positions of a step at position ``t``, in order."""
    if mode == "dense":
        return list(range(t + 1))
    if mode == "diagonal":
        return [min(max(j, 0), t) for j in kept]
    w = n_att - sinks
    return [j for j in range(t + 1) if j < sinks or t - j < w]


def there(entry, pool):
    return 0 <= entry < pool


def update(table, refs, cursor, prompt, lengths, new, most, page, sinks=0, window=0):
    """``page_update`` on lists, in place but for the cursor, which it returns with
    slots, positions, copies and flags.  ``window`` 0: nothing falls behind."""
    pool, width = len(refs), len(table[0])
    batch = len(table)
    for b in range(batch):  # what goes back
        if lengths[b] < 0:
            drop = range(width)
        elif window:
            first, last = prompt[b] + sinks, lengths[b] - window + 1
            drop = [i for i in range(width) if i * page >= first and (i + 1) * page <= last]
        else:
            drop = []
        for i in drop:
            if there(table[b][i], pool):
                refs[table[b][i]] -= 1
            table[b][i] = -1
    wants, fits = [], []
    for b in range(batch):
        n = min(max(new[b], 0), most)
        ok = lengths[b] >= 0 and lengths[b] + n <= width * page
        fits.append(ok)
        want = []
        if ok and n:
            for i in range(lengths[b] // page, (lengths[b] + n - 1) // page + 1):
                e = table[b][i]
                if not there(e, pool):
                    table[b][i] = -1
                    want.append((i, None))
                elif refs[e] > 1:
                    want.append((i, e))
        wants.append(want)
    start = cursor % pool
    free = [g for g in list(range(start, pool)) + list(range(start)) if refs[g] == 0]
    slots = [[-1] * most for _ in range(batch)]
    pos, copies, flags = [-1] * batch, [[-1] * 3 for _ in range(batch)], [0] * batch
    asked = 0
    for b in range(batch):
        if lengths[b] < 0:
            continue
        if not fits[b]:
            flags[b] = TOO_LONG
            continue
        n = min(max(new[b], 0), most)
        asked += len(wants[b])
        if wants[b] and asked > len(free):
            flags[b] = NO_PAGES
            continue
        for k, (i, old) in enumerate(wants[b]):
            g = free[asked - len(wants[b]) + k]
            table[b][i] = g
            refs[g] = 1
            cursor = (g + 1) % pool
            if old is not None:
                refs[old] -= 1
                if k == 0 and i == lengths[b] // page and lengths[b] % page:
                    copies[b] = [old, g, lengths[b] % page]
        for i in range(n):
            r = lengths[b] + i
            slots[b][i] = table[b][r // page] * page + r % page
        pos[b] = max(-1, lengths[b] + n - 1 - prompt[b])
    return cursor, slots, pos, copies, flags


def reorder(table, refs, parent):
    """``page_reorder`` on lists: the new table; ``refs`` changes in place."""
    pool, width = len(refs), len(table[0])
    got = [list(table[p]) if 0 <= p < len(table) else [-1] * width for p in parent]
    for b, p in enumerate(parent):
        for e in got[b]:
            if there(e, pool):
                refs[e] += 1
        for e in table[b]:
            if there(e, pool):
                refs[e] -= 1
    return got


def attention(q, k, v, scale):
    """Output of one query (fp64), scores, and the weighted |v| that bounds its
    rounding; zeros over no rows."""
    if not len(k):
        return np.zeros(v.shape[-1]), np.zeros(0), np.zeros(v.shape[-1])
    z = (k @ q) * scale
    w = np.exp(z - z.max())
    w /= w.sum()
    return w @ v, z, w @ np.abs(v)


def beam(logits, score):
    """``(score, w, v)`` of the best candidates of one request, ``[W, V]`` fp64.  The
    maximum is taken from a logit before anything is added, so that large logits round
    nothing away."""
    beams, vocab = logits.shape
    with np.errstate(all="ignore"):
        x = logits - logits.max(1, keepdims=True)
        z = (x + (score[:, None] - np.log(np.exp(x).sum(1, keepdims=True)))).reshape(-1)
    ok = z > -math.inf  # a NaN is none either
    at = np.flatnonzero(ok)
    # equal scores: the lower beam, its larger logit (rounding makes scores equal), the lower token
    at = at[np.lexsort((at, -logits.reshape(-1)[at], at // vocab, -z[at]))][:beams]
    return [(z[i], int(i) // vocab, int(i) % vocab) for i in at]
