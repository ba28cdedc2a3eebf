"""CPU oracle for drawing and verifying tokens with filters (TEST INFRASTRUCTURE ONLY).

Plain numpy in fp64; nothing in the product path imports this file and this file imports nothing from the product path.

* ``left``    the tokens of one row that temperature, top-k, top-p and min-p leave, walked one by one in the order of falling logits (equal ones by
              their place), and their probabilities.
* ``draw``    the first of them, in vocabulary order, whose running mass exceeds u times the whole.
* ``verify``  one sequence: leading accepted drafts, the next token, the drafts' probabilities.
"""
from __future__ import annotations

import math

import numpy as np


def values(z):
    z = np.asarray(z, np.float64).copy()
    z[np.isnan(z)] = -np.inf
    return np.minimum(z, float(np.finfo(np.float32).max))


def left(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """-> (tokens in vocabulary order, their probabilities); nothing for a row without a finite logit."""
    z = values(z)
    order = sorted((v for v in range(len(z)) if z[v] > -np.inf), key=lambda v: (-z[v], v))
    if not order:
        return np.zeros(0, int), np.zeros(0)
    if not temperature > 0.0 or top_p <= 0.0:
        top_k = 1
        top_p = 1.0
    if not temperature > 0.0:
        temperature = 1.0
    weight = np.exp((z[order] - z[order[0]]) / float(temperature))
    if 0 < top_k < len(z):
        order, weight = order[:top_k], weight[:top_k]
    if top_p < 1.0:
        target, running, n = float(top_p) * math.fsum(weight), 0.0, 0
        while n < len(order) and (n == 0 or running < target):
            running += weight[n]
            n += 1
        order, weight = order[:n], weight[:n]
    if min_p > 0.0:
        keep = weight >= min(float(min_p), 1.0)
        order, weight = [v for v, k in zip(order, keep) if k], weight[keep]
    place = np.argsort(order)
    order, weight = np.asarray(order)[place], weight[place]
    return order, weight / math.fsum(weight)


def draw(tokens, p, u):
    running, total = np.cumsum(p), math.fsum(p)
    at = int(np.searchsorted(running, float(u) * total, side="right"))
    return int(tokens[min(at, len(tokens) - 1)])


def verify(rows, drafts, u_accept, u_sample, **filters):
    """rows [n, V] of one sequence, drafts[i] behind row i (the last counts for nothing) -> accepted, next token, probability of every draft."""
    done = [left(z, **filters) for z in rows]
    p = [float(q[t == d].sum()) if len(t) else 0.0 for (t, q), d in zip(done, drafts)]
    n = 0
    while n < len(rows) - 1 and u_accept[n] < p[n]:
        n += 1
    tokens, q = done[n]
    if n < len(rows) - 1:
        stays = tokens != drafts[n]
        tokens, q = tokens[stays], q[stays]
    return n, (draw(tokens, q, u_sample[n]) if len(tokens) else -1), p
