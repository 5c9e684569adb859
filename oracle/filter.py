"""Oracle: distributions cut by top-k, top-p and min-p, and draws from them.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

A row's tokens are ordered by (logit descending, index ascending); -0.0
equals +0.0, NaN is never kept, -inf is a masked token.  Weights
``w_i = exp((z_i - max z) / T)``.  Top-k keeps the first k tokens, top-p of
these the shortest prefix whose weight is at least p times theirs (at least
one), min-p drops tokens with ``w_i < min_p`` but never the first.  T <= 0 is
the top-1.
"""
from __future__ import annotations

import math

import numpy as np


def top1(z: np.ndarray) -> int:
    """Lowest index of the largest number; 0 when every value is NaN."""
    z = np.where(np.isnan(z), -np.inf, z)
    return int(np.argmax(z)) if np.max(z) > -np.inf else -1


def kept_weights(z, T=1.0, k=0, p=1.0, m=0.0) -> np.ndarray:
    """float64 weights of the kept tokens of one row, 0 elsewhere (all 0 when
    no value is above -inf)."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    V = z.size
    w = np.zeros(V)
    best = top1(z)
    if best < 0:
        return w
    if not T > 0 or k == 1 or z[best] == np.inf:
        w[best] = 1.0
        return w
    fin = np.flatnonzero(np.isfinite(z))
    order = fin[np.lexsort((fin, -z[fin]))]
    ow = np.exp((z[order] - z[order[0]]) / T)
    n = order.size
    if 0 < k < n:
        n = k
    if p < 1:
        # compensated running sums: the oracle's are exact to one rounding
        whole = math.fsum(ow[:n])
        c = np.cumsum(ow[:n].astype(np.longdouble))
        n = min(n, int(np.searchsorted(c, np.longdouble(max(p, 0.0)) * whole, side="left")) + 1)
    if m > 0:
        n = max(1, min(n, int(np.sum(ow >= m))))
    w[order[:n]] = ow[:n]
    return w


def probs(w: np.ndarray) -> np.ndarray:
    s = math.fsum(w)
    return w / s if s > 0 else w


def draw(w: np.ndarray, u: float) -> int:
    """Smallest index whose running weight exceeds u times the whole; the last
    index of positive weight when none does; -1 without any."""
    if not np.any(w > 0):
        return -1
    u = u if u > 0 else 0.0
    c = np.cumsum(w.astype(np.longdouble))
    i = int(np.searchsorted(c, np.longdouble(u) * c[-1], side="right"))
    return min(i, int(np.flatnonzero(w > 0)[-1]))


def sample(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, its probability) of one row."""
    z = np.asarray(z, dtype=np.float64)
    w = kept_weights(z, T, k, p, m)
    t = draw(w, u)
    if t >= 0:
        return t, float(probs(w)[t])
    return no_number(z), 0.0


def no_number(z) -> int:
    """Token of a row without a value above -inf: its lowest index of -inf, 0
    when every value is NaN."""
    masked = np.flatnonzero(np.asarray(z) == -np.inf)
    return int(masked[0]) if masked.size else 0


def accept(pv, qd, d, u, zv=None):
    """(A, final token): pv [B+1, V], qd [B, V] probabilities, d [B] drafts,
    u [B+1] uniforms; zv [B+1, V] the logits of pv, where rows without a value
    above -inf are among them."""
    B, V = qd.shape
    A = 0
    while A < B:
        t = int(d[A])
        if not (0 <= t < V and u[A] * qd[A, t] < pv[A, t]):
            break
        A += 1
    w = pv[A] if A == B else np.maximum(pv[A] - qd[A], 0.0)
    if not np.any(w > 0):
        w = pv[A]
    t = draw(w, u[B])
    return A, t if t >= 0 else 0 if zv is None else no_number(zv[A])
