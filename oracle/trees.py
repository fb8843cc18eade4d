"""Drafts that branch - CPU oracle (test infrastructure only).

Plain numpy in fp64, pure-Python loops; imports nothing from the CUDA package.  A request's new rows are a tree of tokens: row 0 is the pending
token, row i > 0 follows row parent[i] < i.  Siblings are tested in row order.

* ``ancestors`` / ``words``: which rows a row sees, and the same as 64 bits counted back from its own slot;
* ``accept``: speculative sampling with several drafts behind a row.  Drafts that were drawn from q are kept with probability min(1, w(x) / (Z q(x)))
  where w is what the rejections so far have left of p and Z its sum; a rejection leaves max(0, w / Z - q).  Drafts that were chosen (no q) are kept with
  probability w(x) / Z; a rejection leaves w without x.  The token behind the last row kept is drawn from what is left, from p where that is nothing.
  Where p's row, or what a rejection leaves of it, is not finite, no further draft is kept and there is no token;
* ``agree``: the greedy form.

Pinned in ``tests/test_oracle_trees.py``: the emitted distribution is p, chains agree with ``oracle.sampling``, words against ``ancestors``.
"""
from __future__ import annotations

import math

import numpy as np


def ancestors(parent) -> np.ndarray:
    """[n][n] bool: row i sees row j of its request."""
    n = len(parent)
    sees = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parent):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def words(parent):
    """(depths, words) of a request's rows, or None where the words cannot hold it.  Words as Python integers: bit d, the position d before the row's own."""
    n = len(parent)
    if any(not -1 <= p < i for i, p in enumerate(parent)):
        return None
    sees = ancestors(parent)
    out = []
    for i in range(n):
        if not sees[i, :max(0, i - 63)].all():
            return None
        out.append(sum(1 << d for d in range(64) if i - d < 0 or sees[i, i - d]))
    return sees.sum(1) - 1, out


def seen(n_positions: int, own: int, word: int) -> np.ndarray:
    """Which of the positions 0 .. n_positions - 1 the row at position `own` with this word sees."""
    bits = np.array([word >> d & 1 for d in range(64)], dtype=bool)
    back = own - np.arange(n_positions)
    return (back >= 64) | ((back >= 0) & bits[np.clip(back, 0, 63)])


def _draw(w: np.ndarray, u: float) -> int:
    upto = np.cumsum(w)
    at = int(np.searchsorted(upto, u * upto[-1], side="right"))
    return min(at, int(np.flatnonzero(w)[-1]))


def accept(p, q, token, parent, u_accept, u_final):
    """(rows kept, row 0 first; the token behind them) of one request; p [n][V], q [n][V] or None."""
    p = np.asarray(p, dtype=np.float64)
    q = None if q is None else np.asarray(q, dtype=np.float64)
    n, V = p.shape
    passed = [i > 0 and not (0 <= parent[i] < i and 0 <= token[i] < V) for i in range(n)]
    kept = [0]
    while True:
        node = kept[-1]
        w, z, go = p[node].copy(), 1.0, None
        for c in range(node + 1, n):
            if passed[c] or parent[c] != node:
                continue
            x = token[c]
            if float(u_accept[c]) * z * (1.0 if q is None else q[node, x]) < w[x]:
                go = c
                break
            if q is None:
                w[x] = 0.0
            elif z > 0:
                w = np.maximum(w / z - q[node], 0.0)
            z = math.fsum(w) if np.isfinite(p[node]).all() and np.isfinite(w).all() else math.nan
            if math.isnan(z):
                break
        if go is None:
            break
        kept.append(go)
    if math.isnan(z) or not np.isfinite(p[kept[-1]]).all():
        return kept, -1
    if not w.any():
        w = p[kept[-1]]
    return kept, (_draw(w, float(u_final)) if w.any() else -1)


def agree(best, token, parent):
    """(rows kept, next token), greedily."""
    kept = [0]
    while True:
        node = kept[-1]
        go = next((c for c in range(node + 1, len(token)) if parent[c] == node and token[c] == best[node]), None)
        if go is None:
            return kept, best[node]
        kept.append(go)
