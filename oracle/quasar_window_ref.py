"""CPU oracle for windows over a paged cache and for other rotary positions (TEST INFRASTRUCTURE ONLY).

Plain numpy; nothing in the product path imports this file and this file imports nothing from the product path.

* ``sees``       whether the row at a position sees another: not behind it, and within the window or among the first tokens.
* ``attention``  rows of one sequence behind `length` cached positions: what each sees, one row at a time, in fp64.
* ``trim``       the table's pages of which no position is seen from the next position on, asked position by position.
* ``rotate``     the first `dims` elements of heads as complex numbers, turned; fp64.
"""
from __future__ import annotations

import numpy as np

D = 128


def sees(row: int, pos: int, window: int, sinks: int) -> bool:
    return pos <= row and (row - pos < window or pos < sinks)


def attention(q, k, v, length: int, window: int, sinks: int):
    """q [n, Hq, 128], k, v [total >= length + n, Hkv, 128] fp64 -> (out [n, Hq, 128], sum of weight * |value| likewise)."""
    n, hq, _ = q.shape
    g = hq // k.shape[1]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(n):
        row = length + i
        seen = np.unique(np.r_[0:min(sinks, row + 1), max(0, row - window + 1):row + 1]).astype(int)
        ks, vs = k[seen], v[seen]
        for h in range(hq):
            s = ks[:, h // g] @ q[i, h] / np.sqrt(D)
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], size[i, h] = w @ vs[:, h // g], w @ np.abs(vs[:, h // g])
    return out, size


def trim(refs, lengths, table, page_len: int, window: int, sinks: int):
    refs, table = list(refs), [list(r) for r in table]
    for row, length in zip(table, lengths):
        for c, page in enumerate(row):
            # (rows further on see less of what is cached: the next one decides, and a page may hold positions behind it)
            first, last = c * page_len, (c + 1) * page_len - 1
            wanted = last >= length or first < sinks or any(sees(length, p, window, sinks) for p in {first, last})
            if page >= 0 and not wanted:
                refs[page] -= 1
                row[c] = -1
    return refs, table


def rotate(x, pos, freq, layout: str, magnitude: float = 1.0):
    """x [rows, heads, 128] fp64, pos [rows], freq [dims / 2] radians a position."""
    x, half = np.array(x, np.float64), len(freq)
    turn = magnitude * np.exp(1j * np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64))[:, None]
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = (x[..., a] + 1j * x[..., b]) * turn
    x[..., a], x[..., b] = z.real, z.imag
    return x
