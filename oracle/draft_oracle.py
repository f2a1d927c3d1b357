"""Float64 CPU oracle of drafting over the paged cache (test infrastructure only): the definitions, one token at a time."""
from __future__ import annotations

import numpy as np


def freqs(rot_dim, base=10000.0, kind="plain", factor=1.0, context=0.0, low=1.0, high=32.0):
    out = []
    for i in range(rot_dim // 2):
        if kind == "base":
            f = (base * factor ** (rot_dim / max(rot_dim - 2, 1))) ** (-2 * i / rot_dim)
        else:
            f = base ** (-2 * i / rot_dim)
        if kind == "linear":
            f = f / factor
        if kind == "parts":
            turns = context * f / (2 * np.pi)
            g = min(max((turns - low) / (high - low), 0.0), 1.0)
            f = g * f + (1 - g) * f / factor
        out.append(f)
    return np.array(out)


def pairs_of(rot_dim, halves):
    i = np.arange(rot_dim // 2)
    return (i, rot_dim // 2 + i) if halves else (2 * i, 2 * i + 1)


def rotate(x, pos, f, halves=True, magnitude=1.0, back=False):
    """x [n, H, d] -> the rotated heads, and reach [n, H, d]: magnitude (|a| + |b|) of each element's pair, 0 where nothing is rotated."""
    x = np.asarray(x, dtype=np.float64)
    y, reach = x.copy(), np.zeros_like(x)
    a, b = pairs_of(2 * len(f), halves)
    for t in range(x.shape[0]):
        angle = (np.longdouble(int(pos[t])) * f.astype(np.longdouble)) * (-1 if back else 1)
        c, s = (np.float64(magnitude) * fn(angle).astype(np.float64) for fn in (np.cos, np.sin))
        p, q = x[t][:, a], x[t][:, b]
        y[t][:, a], y[t][:, b] = p * c - q * s, p * s + q * c
        reach[t][:, a] = reach[t][:, b] = magnitude * (np.abs(p) + np.abs(q))
    return y, reach


def path_to(parent, i):
    """Node i's ancestors and itself, root first.  Numbers that are no earlier node stand for -1."""
    out = []
    while i >= 0:
        out.append(i)
        p = int(parent[i])
        i = p if 0 <= p < i else -1
    return out[::-1]


def attention(q, k, v, scale, parent):
    """q [n, Hq, d], the nodes of a draft, k and v [Hk, L, d] with the draft's tokens last -> out, lse, spread, reach as
    paged_oracle.attention gives them."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, Hq, d = q.shape
    Hk, L, _ = k.shape
    out, spread = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, reach = np.full((Hq, n), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        keys = list(range(max(0, L - n))) + [L - n + a for a in path_to(parent, i) if L - n + a >= 0]
        if not keys:
            continue
        kk, vv, qq = k[:, keys], v[:, keys], q[i].reshape(Hk, Hq // Hk, d)
        x = scale * (qq @ kk.transpose(0, 2, 1))             # [Hk, heads of the group, keys]
        m = x.max(axis=2, keepdims=True)
        m = np.where(np.isfinite(m), m, 0.0)
        p = np.exp(x - m)
        z = p.sum(axis=2, keepdims=True)
        seen = (z > 0.0) | np.isnan(z)
        with np.errstate(invalid="ignore", divide="ignore"):
            out[i] = np.where(seen, p @ vv / z, 0.0).reshape(Hq, d)
            spread[i] = np.where(seen, p @ np.abs(vv) / z, 0.0).reshape(Hq, d)
            lse[:, i] = np.where(seen, m + np.log(z), -np.inf).reshape(Hq)
        reach[i] = abs(scale) * (np.abs(qq) @ np.abs(kk).transpose(0, 2, 1)).max(axis=2).reshape(Hq)
    return out, lse, spread, reach


def plan(table, kv_len, refs, rows, add, ps, total, parent=None, pruned=None):
    """In place; returns cu, slot, pos."""
    n_rows, width = table.shape
    cu, slot, pos = [0], [-1] * total, [-1] * total
    free = [int(p) for p in np.flatnonzero(refs == 0)]
    open_, room, seen = True, True, set()
    for r, x in zip(rows, add):
        r, x = int(r), int(x)
        first = cu[-1]
        room = room and first + max(x, 0) <= total
        cu.append(first + max(x, 0) if room else first)
        if not room or not 0 <= r < n_rows or x < 0 or r in seen or not 0 <= kv_len[r] <= width * ps - x:
            continue
        seen.add(r)
        old = int(kv_len[r])
        have, want = -(-old // ps), -(-(old + x) // ps)
        open_ = open_ and want - have <= len(free)
        if open_:
            for t in range(have, want):
                table[r, t] = free.pop(0)
                refs[table[r, t]] = 1
            kv_len[r] = old + x
        for i in range(x):
            at = old + i
            if open_:
                slot[first + i] = int(table[r, at // ps]) * ps + at % ps
            deep = i if parent is None else len(path_to(parent[first:first + x], i)) - 1
            pos[first + i] = old + deep + (int(pruned[r]) if pruned is not None else 0)
    return np.array(cu), np.array(slot), np.array(pos)


def accept(table, kv_len, refs, layers, rows, counts, paths, ps):
    """In place; layers: list of (k_pages, v_pages) [n_pages, Hk, ps, d]; paths: each row's nodes, ascending."""
    for r, m, path in zip(rows, counts, paths):
        L = int(kv_len[r])
        base = L - m
        for t, node in enumerate(path):
            a, b = base + node, base + t
            for pages in [x for kv in layers for x in kv]:
                pages[table[r, b // ps], :, b % ps] = pages[table[r, a // ps], :, a % ps]
        for t in range(-(-(base + len(path)) // ps), -(-L // ps)):
            refs[table[r, t]] -= 1
        kv_len[r] = base + len(path)
