"""Float64 CPU oracle of the paged cache and its attention (test infrastructure only): the definitions, one sequence, one
token at a time."""
from __future__ import annotations

import numpy as np


def gather(pages, table_row, length):
    """Tokens 0 .. length-1 of a row: [Hk, length, d] from pages [n_pages, Hk, page_size, d]."""
    ps = pages.shape[2]
    t = np.arange(length)
    return pages[np.asarray(table_row)[t // ps], :, t % ps].transpose(1, 0, 2)


def attention(q, k, v, scale, causal):
    """q [n, Hq, d], k and v [Hk, L, d] -> out [n, Hq, d], lse [Hq, n], and for error bounds spread [n, Hq, d] = sum p |v| / z
    and reach [n, Hq] = max |scale| sum |q_e k_e| over the keys that the row sees (0 where it sees none)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, Hq, d = q.shape
    Hk, L, _ = k.shape
    out, spread = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, reach = np.full((Hq, n), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        lim = min(L, max(0, L - n + i + 1)) if causal else L
        if lim == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hk)
            x = scale * (k[g, :lim] @ q[i, h])
            m = x.max()
            p = np.exp(x - m) if np.isfinite(m) else np.exp(x - (0.0 if m == -np.inf else m))
            z = p.sum()
            if z == 0.0:
                continue
            out[i, h] = p @ v[g, :lim] / z
            spread[i, h] = p @ np.abs(v[g, :lim]) / z
            lse[h, i] = (m if np.isfinite(m) else 0.0) + np.log(z)
            reach[i, h] = abs(scale) * (np.abs(k[g, :lim]) @ np.abs(q[i, h])).max()
    return out, lse, spread, reach


def grow(table, kv_len, refs, rows, add, ps):
    """In place: the lowest free pages in the order of the list; a row that does not get all stops the list."""
    free = [int(p) for p in np.flatnonzero(refs == 0)]
    for r, a in zip(rows, add):
        have, want = -(-int(kv_len[r]) // ps), -(-(int(kv_len[r]) + int(a)) // ps)
        if want - have > len(free):
            break
        for t in range(have, want):
            table[r, t] = free.pop(0)
            refs[table[r, t]] = 1
        kv_len[r] += a


def fork(table, kv_len, refs, layers, parents, children):
    """In place; layers: list of (k_pages, v_pages)."""
    ps = layers[0][0].shape[2] if layers else None
    return fork_tables(table, kv_len, refs, parents, children, ps, layers)


def fork_tables(table, kv_len, refs, parents, children, ps, layers=()):
    for a, b in zip(parents, children):
        full, part = divmod(int(kv_len[a]), ps)
        if part:
            free = np.flatnonzero(refs == 0)
            if free.size == 0:
                break
            table[b, full] = free[0]
            refs[free[0]] = 1
            for k, v in layers:
                k[free[0], :, :part] = k[table[a, full], :, :part]
                v[free[0], :, :part] = v[table[a, full], :, :part]
        table[b, :full] = table[a, :full]
        np.add.at(refs, table[a, :full], 1)
        kv_len[b] = kv_len[a]


def free(table, kv_len, refs, rows, ps):
    for r in rows:
        np.subtract.at(refs, table[r, :-(-int(kv_len[r]) // ps)], 1)
        kv_len[r] = 0


def write(pages, table, kv_len, rows, counts, values):
    """In place: values[i] [Hk, counts[i], d] become the last tokens of row rows[i]."""
    ps = pages.shape[2]
    for r, n, x in zip(rows, counts, values):
        t = np.arange(int(kv_len[r]) - n, int(kv_len[r]))
        pages[table[r][t // ps], :, t % ps] = np.asarray(x).transpose(1, 0, 2)
