"""CPU oracle for a batch of sequences over a paged key/value cache (TEST INFRASTRUCTURE ONLY).

Plain numpy and Python; nothing in the product path imports this file and this file imports nothing from the product path.
Sequences are lists of rows, books are walked one sequence and one page at a time, attention is the definition in fp64.

* ``block_places``   where (position in a block of 32, d) lies in a page's block of keys and of values (include/quasar.h).
* ``e4m3_to_f64``, ``f64_to_e4m3``   the 8-bit type: 4 exponent bits of bias 7, 3 fraction bits, 0x7F / 0xFF = NaN, largest 448;
                     rounding to nearest, ties to even, saturating.
* ``Books``          refs, lengths and table with reserve, fork and compact.
* ``attention``      rows of one sequence behind `length` cached positions: causal, grouped heads, softmax of q.k / sqrt(128).
"""
from __future__ import annotations

import numpy as np

D, BLOCK = 128, 32


def block_places(kv: str):
    """(keys, values): [32, 128] element offsets in a block."""
    keys, values = np.empty((BLOCK, D), np.int64), np.empty((BLOCK, D), np.int64)
    for p in range(BLOCK):
        for d in range(D):
            if kv == "bf16":
                keys[p, d] = np.ravel_multi_index((p // 16, d // 32, d % 32 // 8, p % 16, d % 8), (2, 4, 4, 16, 8))
                values[p, d] = np.ravel_multi_index((d // 16, p % 16 // 4, d % 16, p // 16, p % 4), (8, 4, 16, 2, 4))
            else:
                keys[p, d] = np.ravel_multi_index((p // 16, d // 64, d % 32 // 8, p % 16, d // 32 % 2, d % 8), (2, 2, 4, 16, 2, 8))
                values[p, d] = np.ravel_multi_index((d // 32, p % 16 // 4, d % 16, d // 16 % 2, p // 16, p % 4), (4, 4, 16, 2, 2, 4))
    return keys, values


def e4m3_to_f64(codes) -> np.ndarray:
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    mag = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    mag = np.where((c & 0x7F) == 0x7F, np.nan, mag)
    return np.where(c & 0x80, -mag, mag)


def f64_to_e4m3(x) -> np.ndarray:
    x = np.asarray(x, np.float64)
    grid = e4m3_to_f64(np.arange(0x7F))                        # 0 .. 448, ascending: index = code
    a = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(grid, a)
    lo = np.maximum(hi - 1, 0)
    below, above = a - grid[lo], grid[hi] - a
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def attention(q, k, v, length: int):
    """q [n, Hq, 128], k, v [total >= length + n, Hkv, 128] fp64 -> (out [n, Hq, 128], sum of weight * |value| likewise)."""
    n, hq, _ = q.shape
    g, total = hq // k.shape[1], length + n
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    hidden = np.arange(total)[None, :] > length + np.arange(n)[:, None]
    for h in range(hq):
        s = q[:, h] @ k[:total, h // g].T / np.sqrt(D)
        s[hidden] = -np.inf
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        out[:, h] = w @ v[:total, h // g]
        size[:, h] = w @ np.abs(v[:total, h // g])
    return out, size


class Books:
    """The books of a cache, walked one entry at a time.  `copies`: (from, to, blocks) of the last call."""

    def __init__(self, refs, lengths, table, page_len: int):
        self.refs, self.lengths, self.table, self.page_len = [int(r) for r in refs], [int(n) for n in lengths], [[int(i) for i in row] for row in table], page_len
        self.copies = []

    def reserve(self, n_new):
        self.copies, status, short = [], [], False
        for s, n in enumerate(n_new):
            n, row, length = int(n), self.table[s], self.lengths[s]
            if n <= 0:
                status.append(1)
                continue
            first, need = length // self.page_len, -(-(length + n) // self.page_len)
            if need > len(row):
                status.append(0)
                continue
            free = [i for i, r in enumerate(self.refs) if r == 0]
            last = row[first]
            copy = length % self.page_len != 0 and last >= 0 and self.refs[last] > 1
            wanted = [c for c in range(first, need) if row[c] < 0 or (copy and c == first)]
            if short or len(wanted) > len(free):
                short = True
                status.append(0)
                continue
            for c, page in zip(wanted, free):
                row[c] = page
                self.refs[page] = 1
            if copy:
                self.refs[last] -= 1
                self.copies.append((last, row[first], -(-(length % self.page_len) // BLOCK)))
            status.append(1)
        return status

    def fork(self, parent, keep=None):
        old, lengths, n = [list(r) for r in self.table], list(self.lengths), len(self.table)
        for s in range(n):
            p = int(parent[s])
            length = lengths[p] if 0 <= p < n else 0
            if keep is not None:
                length = min(length, int(keep[s]))
            length = max(length, 0)
            held = -(-length // self.page_len)
            row = [old[p][c] if c < held else -1 for c in range(len(old[s]))] if 0 <= p < n else [-1] * len(old[s])
            for page in row:
                if page >= 0:
                    self.refs[page] += 1
            for page in old[s]:
                if page >= 0:
                    self.refs[page] -= 1
            self.table[s], self.lengths[s] = row, length

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        to = list(range(len(self.refs)))
        holes = [i for i in range(n) if self.refs[i] <= 0]
        moved = [i for i in range(n, len(self.refs)) if self.refs[i] > 0]
        self.copies = [(src, dst, self.page_len // BLOCK) for src, dst in zip(moved, holes)]
        for src, dst in zip(moved, holes):
            to[src] = dst
            self.refs[dst], self.refs[src] = self.refs[src], 0
        self.table = [[to[i] if i >= 0 else i for i in row] for row in self.table]
        return to
