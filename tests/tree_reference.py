"""Plain reference of the speculative-decoding operators, on the CPU in 64 bits: attention of drafted trees with the
error bounds that follow from the kernels' roundings, verification, and what a commit leaves in the pages."""
from __future__ import annotations

import math

import numpy as np

from tests import paged_reference as R


def random_tree(rng, T, width=3):
    """Parents of T nodes, a parent before its children; -1 for node 0."""
    return np.array([-1] + [int(rng.integers(max(0, j - 2 * width), j)) for j in range(1, T)], dtype=np.int32)


def ancestors(parents):
    """[T][T]: node i sees node j."""
    T = len(parents)
    sees = np.zeros((T, T), dtype=bool)
    for i in range(T):
        up = i
        while up >= 0:
            sees[i, up] = True
            up = int(parents[up])
    return sees


def visible(parents, length):
    """Context tokens that each node sees, as lists of indexes; none for a node whose own token is negative."""
    T, c = len(parents), length - len(parents)
    sees = ancestors(parents)
    return [[] if c + i < 0 else list(range(max(0, c))) + [c + j for j in range(T) if sees[i, j] and c + j >= 0] for i in range(T)]


def attend(q, k, v, scale, fmt):
    """q [Hq][D], k and v [tokens][Hkv][D] of the tokens that a node sees -> out, lse and the bounds of both.

    Roundings of paged_reference.attend, and in the 4-bit format those of operands in f16: a key is exact, as a product and what
    its rounding left, down to 2^-25 for each; a query element is exact down to 2^-17 of the row's largest and within 2^-25
    of that below.  They change a score by at most scale times the sums below, and the
    probabilities by that."""
    out, lse, tol, lse_tol = R.attend(q, k, v, scale, fmt)
    if fmt == "bf16" or len(k) == 0:
        return out, lse, tol, lse_tol
    Hkv = k.shape[1]
    kk, vv = (np.repeat(x, q.shape[0] // Hkv, axis=1) for x in (k, v))
    aq, ak = np.abs(q), np.abs(kk)
    top = aq.max(-1)
    more = 2.0 ** -24 * aq.sum(-1) + 2.0 ** -25 * top * ak.sum(-1)
    more = 1.01 * scale * more.max(0)
    s = np.einsum("hd,thd->ht", q, kk) * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    mass = np.einsum("ht,thd->hd", p / p.sum(-1, keepdims=True), np.abs(vv))
    return out, lse, tol + (1 + 2.0 ** -7) * np.expm1(2 * more)[:, None] * mass, lse_tol + more


def verify(target, draft, tokens, parents, u_accept, u_next):
    """One request: rows [T][V] -> (path, next token)."""
    T = len(tokens)
    if T == 0:
        return [], -1

    def row(x, i):
        x = np.asarray(x[i], dtype=np.float64)
        return np.where(x > 0, x, 0.0)

    V = len(target[0])
    path, cur, p, z = [0], 0, row(target, 0), 1.0
    for j in range(1, T):
        x = int(tokens[j])
        if parents[j] != cur or not 0 <= x < V:
            continue
        q = None if draft is None else row(draft, cur)
        if p[x] > 0 and float(u_accept[j]) * (1.0 if q is None else q[x]) * z < p[x]:
            path.append(j)
            cur, p, z = j, row(target, j), 1.0
        elif q is None:
            z -= p[x]
            p[x] = 0.0
        else:
            left = np.maximum(p / z - q, 0.0)
            total = math.fsum(left)
            if total > 0:
                p, z = left, total
    goal = float(u_next) * math.fsum(p)
    there = np.flatnonzero(p > 0)
    if len(there) == 0:
        return path, -1
    over = there[np.cumsum(p[there]) > goal]
    return path, int(over[0] if len(over) else there[-1])
