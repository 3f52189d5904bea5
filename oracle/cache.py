"""The operators around a paged key-value cache, from their definitions: whole numbers with plain loops, values in 64 bits
(numpy).  Test infrastructure only; shares nothing with the HIP library."""
from __future__ import annotations

import numpy as np


def assign(page, cached, fresh, table, free, n_tokens):
    """-> (table after, begin, length, slot, position, owner, taken); the free list's pages are handed out request by request."""
    table = np.array(table)
    width = table.shape[1]
    begin, slot, position, owner, length, taken = [0], [], [], [], [], 0
    for r, f in enumerate(fresh):
        c, f = max(int(cached[r]) if cached is not None else 0, 0), max(int(f), 0)
        for j in range(min(-(-c // page), width), min(-(-(c + f) // page), width)):
            table[r, j] = free[taken] if taken < len(free) else -1
            taken += 1
        for at in range(c, c + f):
            j = at // page
            p = table[r, j] if j < width else -1
            slot.append(int(p) * page + at % page if p >= 0 else -1)
            position.append(at)
            owner.append(r)
        begin.append(begin[-1] + f)
        length.append(c + f)
    for x in (slot, position, owner):
        x += [-1] * (n_tokens - len(x))
    return table, begin, length, slot[:n_tokens], position[:n_tokens], owner[:n_tokens], taken


def turn(x, position, freq, axis_pairs, interleaved=False, inverse=False):
    """x [tokens, heads, dim] float64; position [axes, tokens]; freq float32."""
    y = np.array(x, dtype=np.float64)
    pairs, p = len(freq), 0
    for a, n in enumerate(axis_pairs):
        for _ in range(n):
            i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)
            angle = position[a].astype(np.float64) * np.float64(freq[p])
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
            y[:, :, i] = x[:, :, i] * c - x[:, :, j] * s
            y[:, :, j] = x[:, :, j] * c + x[:, :, i] * s
            p += 1
    return y


def attend(q, k, v, table, length, page, scale, window=0):
    """q [requests, heads, dim], k and v [pages, page, kv_heads, dim], float64 -> (out, lse, sum of p |v|, the largest sum of |q k| of a
    score of the row).  Rows that see nothing, or nothing over -inf: 0 and -inf."""
    n, heads, dim = q.shape
    group, width = heads // k.shape[2], table.shape[1]
    out, mass = np.zeros_like(q), np.zeros_like(q)
    lse, most = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for r in range(n):
        last = min(max(int(length[r]), 0), width * page)
        seen = [i for i in range(max(last - window, 0) if window else 0, last) if 0 <= table[r, i // page] < k.shape[0]]
        if not seen:
            continue
        pages, rows = [table[r, i // page] for i in seen], [i % page for i in seen]
        for h in range(heads):
            kh, vh = k[pages, rows, h // group], v[pages, rows, h // group]
            with np.errstate(all="ignore"):
                s = scale * (kh * q[r, h]).sum(1)
                top = s.max()
                if top == -np.inf:
                    continue
                e = np.exp(s - top)
                out[r, h] = (e[:, None] * vh).sum(0) / e.sum()
                mass[r, h] = (e[:, None] * np.abs(vh)).sum(0) / e.sum()
                lse[r, h] = top + np.log(e.sum())
                most[r, h] = abs(scale) * np.abs(kh * q[r, h]).sum(1).max()
    return out, lse, mass, most
