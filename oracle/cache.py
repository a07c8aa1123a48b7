"""Plain definitions of the paged cache's operators, in numpy and 64 bits.

Block tables and slot maps from request lengths, the append of records, and
attention over the paged cache: one request, one row and one head at a time.
"""

from __future__ import annotations

import numpy as np


def tables_build(cached, added, n_slots, groups):
    """groups: dicts with block_tokens, free (ids in order), tables (int [requests, stride]) or None, slots (bool).

    Returns starts, lens, result, and per group (tables, slots).
    """
    n = len(cached)
    admitted, rows, taken = 0, 0, [0] * len(groups)
    starts, plan = [], []
    for r in range(n):
        c, a = int(cached[r]), int(added[r])
        if c < 0 or a < 0 or c + a >= 2 ** 31 or rows + a > n_slots:
            break
        need = []
        for g in groups:
            if g["tables"] is None:
                need.append((0, 0))
                continue
            B = g["block_tokens"]
            need.append((-(-c // B), -(-(c + a) // B)))
        if any(g["tables"] is not None and (k > g["tables"].shape[1] or t + k - h > len(g["free"]))
               for g, (h, k), t in zip(groups, need, taken)):
            break
        starts.append(rows)
        plan.append([(h, k, t) for (h, k), t in zip(need, taken)])
        rows += a
        taken = [t + k - h for t, (h, k) in zip(taken, need)]
        admitted += 1
    starts += [rows] * (n + 1 - admitted)
    lens = [int(c) + int(a) if r < admitted else max(0, int(c)) for r, (c, a) in enumerate(zip(cached, added))]
    out = []
    for gi, g in enumerate(groups):
        if g["tables"] is None:
            out.append((None, None))
            continue
        B, tables = g["block_tokens"], g["tables"].copy()
        slots = np.full(n_slots, -1, np.int64)
        for r in range(admitted):
            h, k, t = plan[r][gi]
            tables[r, h:k] = g["free"][t:t + k - h]
            for i in range(int(added[r])):
                at = int(cached[r]) + i
                b = int(tables[r, at // B])
                slots[starts[r] + i] = b * B + at % B if b >= 0 else -1
        out.append((tables, slots if g["slots"] else None))
    return np.array(starts, np.int32), np.array(lens, np.int32), np.array([admitted] + taken, np.int64), out


def scale_of(x):
    """The fp32 scale of a planar record of fp32 values."""
    x = np.asarray(x, np.float32)
    if not np.all(np.isfinite(x)):
        return np.float32(np.nan)
    return np.float32(np.max(np.abs(x)) / np.float32(448))


def visible(mode, n, T, i, *, mask=None, window=0, prefix=0, document=0):
    """bool [n]: the keys that row i of a request of n tokens and T rows sees; and the row's position."""
    base = n - T
    j = np.arange(n)
    if mode == "tree":
        bits = [k for k in range(64 * len(mask)) if int(mask[k // 64]) >> (k % 64) & 1]
        p = base + len(bits) - 1
        see = j < base
        if window:
            see &= j > p - window
        for k in bits:
            if k < T and base + k >= 0:
                see[base + k] = True
        return see, p
    p = base + i
    see = (j <= p) | (j < min(prefix, n))
    if window:
        see &= j > p - window
    return see & (j >= document), p


def attend(q, k, v, see, p, scale, cap=0.0, slope=0.0):
    """One row and head: q [dk], k [n, dk], v [n, dv], float64.

    Returns out, lse, and what bounds its error: the sum of weight * |v| and
    the largest sum of |q k| * scale of a key that the row sees.
    """
    at = np.nonzero(see)[0]
    if not len(at):
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        s = k[at] @ q * scale
        if cap:
            s = cap * np.tanh(s / cap)
        s = s - slope * np.abs(p - at)
        top = s.max()
        w = np.exp(s - top)
        total = w.sum()
        w = w / total
        return w @ v[at], top + np.log(total), w @ np.abs(v[at]), float((np.abs(k[at]) @ np.abs(q)).max() * scale)
