"""Several new tokens of a request at once, in plain slow fp64.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

Node ``i`` of a tree of new tokens stands at decode position ``base +
depth(i)``; position ``j < 0`` is prompt row ``L_p + j``.  It attends every
cached position and every ancestor (and itself) that its mode keeps in reach:
all of them in dense mode; in window mode the ``S`` sinks (prompt rows
included) and the ``W = N_att - S`` most recent positions.
"""

from __future__ import annotations

import numpy as np

from .fp8 import decode_e4m3


def line(parents, i):
    """Node ``i`` and its ancestors, the topmost first."""
    at = [i]
    while parents[at[-1]] >= 0:
        at.append(parents[at[-1]])
    return at[::-1]


def chain(n):
    return list(range(-1, n - 1))


def reach(p, j, sinks, window):
    """Whether a token at position ``p`` attends position ``j <= p``."""
    return window is None or j < sinks or p - j < window


def keys_of(parents, i, base, prompt, sinks, window):
    """(cached positions, nodes) that node ``i`` attends."""
    up = line(parents, i)
    p = base + len(up) - 1
    return ([j for j in range(-prompt, base) if reach(p, j, sinks, window)],
            [m for e, m in enumerate(up) if reach(p, base + e, sinks, window)])


def attend(q, k, v, scale):
    """``softmax(scale q k) v`` of ``q [d]`` over ``k, v [n, d]``, and a bound
    of what fp32 arithmetic (sums of ``n`` terms and of ``d`` products in any
    order, one exponential per key) may be off by, as a multiple of the
    largest ``|v|``.

    Each of the d products is exact in fp32; their sum is off by at most
    d 2^-24 sum|q k|, the scaled difference from the maximum by one rounding of
    each of its two terms and of the scale (at most 4 2^-24 max|s|), the
    exponential by 2^-22, and both sums of the n terms by n 2^-24.  A weight's
    relative error enters the quotient twice."""
    s = scale * (k @ q)
    z = s - s.max()
    w = np.exp(z)
    out = (w / w.sum()) @ v
    dots = abs(scale) * (np.abs(k) @ np.abs(q)).max()
    eps = 2.0 ** -24
    band = 2 * (len(q) * eps * dots + 4 * eps * np.abs(s).max() + 4 * eps) + 2 * (len(k) + 4) * eps
    return out, band


def verify(parents, tokens, target, draft, uniform, count):
    """(accepted nodes, next token) by rejection sampling; ``draft`` None:
    every drafted token is certain."""
    if count == 0:
        return [], -1
    clean = lambda x: np.where(x > 0, x, 0.0).astype(np.float64)  # noqa: E731
    vocab = target.shape[1]
    path = [0]
    while True:
        c = path[-1]
        p, mass, spent = clean(target[c]), 1.0, False
        q = None if draft is None else clean(draft[c])
        for i in [i for i in range(c + 1, count) if parents[i] == c]:
            x, u = int(tokens[i]), float(uniform[i])
            have = p[x] if 0 <= x < vocab else 0.0
            if q is not None:
                prop = q[x] if 0 <= x < vocab else 0.0
                if not spent and u * prop * mass < have:
                    path.append(i)
                    break
                left = np.maximum(p / mass - q, 0.0)
                if left.sum() > 0 and not spent:
                    p, mass = left, left.sum()
                else:
                    spent = True
            else:
                if have > 0 and u * mass < have:
                    path.append(i)
                    break
                if 0 <= x < vocab:
                    mass -= have
                    p = p.copy()
                    p[x] = 0.0
        if path[-1] == c:
            break
    upto = np.cumsum(p)
    if not upto[-1] > 0:
        return path, -1
    over = np.nonzero(upto > float(uniform[-1]) * upto[-1])[0]
    return path, int(over[0] if len(over) else np.nonzero(p)[0][-1])


_CODES = np.arange(0x7F)  # the non-negative finite values, ascending
_VALUES = decode_e4m3(_CODES)


def encode_e4m3(x):
    """Nearest E4M3 byte of fp32 values (ties to the even code, clamped to +-448)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.minimum(np.searchsorted(_VALUES, a, side="left"), 0x7E)
    lo = np.maximum(hi - 1, 0)
    to_lo, to_hi = a - _VALUES[lo], _VALUES[hi] - a
    code = np.where(to_lo < to_hi, lo, np.where(to_hi < to_lo, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), 0x7F, code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)
