"""Values by which every block of 32 positions of a long context shows in the attention's output, and how near that has to be.

Random values average out: over 30000 positions a block more or less changes an output by less than its roundings may.  Here block b adds to
column b % 128 alone, so that a column is a sum over few blocks, all of one sign, and a block that is left out, or taken twice, changes its
column by a large part of it."""
import numpy as np

from oracle import quasar_paged_ref as pg

D, BLOCK = 128, 32


def block_values(total):
    """[total, 128]: 1, 2 or 4 in the column of the position's block, else 0 (exact in both types of pages)."""
    block = np.arange(total) // BLOCK
    v = np.zeros((total, D))
    v[np.arange(total), block % D] = 2.0 ** (block // D % 3)
    return v


def attention_and_bound(q, k, v, length, kv):
    """(out, tolerance) [n, Hq, 128].  As Batch.expected, but with the roundings of each type of pages: weights to bf16 (2^-8 relatively), or, for
    e4m3 pages, to fp16 (2^-11, and 2^-31 of the largest where that is below fp16's normal range), their sum being that of the rounded ones."""
    out, size = pg.attention(q, k, v, length)
    most = np.linalg.norm(q, axis=2).max() * np.linalg.norm(k, axis=2).max() / np.sqrt(D)          # >= sum |q k| / sqrt(128)
    weight = 2.0 ** -8 if kv == "bf16" else 2.0 ** -11
    tol = 2.0 ** -8 * np.abs(out) + (2 * weight + 4 * 132 * 2.0 ** -24 * most) * size
    if kv != "bf16":
        tol = tol + 2.0 ** -31 * np.repeat(np.abs(v).sum(axis=0), q.shape[1] // k.shape[1], axis=0)[None]
    return out, 1.01 * tol + 1e-30
