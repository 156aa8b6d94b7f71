"""Plain CPU oracle of sampling: a query's scores, and the token that given random numbers draw from them.

TEST INFRASTRUCTURE ONLY (see pced_oracle). NumPy and the plain definitions, one query and one filter at a time, weights in
extended precision.
"""
from __future__ import annotations

import math

import numpy as np


def scores(rows, beta, prior, allowed=None, real=np.float32):
    """S [V] (-inf: no candidate) and the best expert [V] (1 on; 0: none) of adjusted rows [N + 1][V] by Eq. 2, every
    operation rounded to `real`."""
    rows = np.asarray(rows, dtype=real)
    best, who = np.full(rows.shape[1], -np.inf, dtype=real), np.zeros(rows.shape[1], np.int64)
    with np.errstate(all="ignore"):
        for k, (b, c) in enumerate(zip(beta, prior)):
            f = ((real(1) + real(b)) * rows[k + 1] - real(b) * rows[0]) + real(c)
            up = f > best  # (not of NaN)
            if allowed is not None:
                up &= np.asarray(allowed)
            best, who = np.where(up, f, best), np.where(up, k + 1, who)
    return best, who


def sample(S, temperature, u, top_k=0, top_p=1.0, min_p=0.0):
    """(token, ln of its share, tokens kept) from scores S; (-1, -inf, 0) without a candidate."""
    S = np.asarray(S, dtype=np.float64)
    order = [v for v in np.argsort(-S, kind="stable") if S[v] > -np.inf]  # equal scores: the lower token first
    if not order:
        return -1, -math.inf, 0
    greedy = not temperature > 0
    T = np.longdouble(1.0 if greedy else min(temperature, np.finfo(np.float32).max))
    s = S[order].astype(np.longdouble)
    with np.errstate(invalid="ignore"):
        z = np.where(s == s[0], np.longdouble(0), (s - s[0]) / T)
    n = 1 if greedy else len(order) if top_k <= 0 else min(top_k, len(order))
    w = np.exp(z)
    if top_p < 1 and not greedy:
        run = np.cumsum(w[:n])
        n = 1 + int((run < np.longdouble(max(top_p, 0.0)) * run[-1]).sum())
    if min_p > 0 and not greedy:
        n = min(n, max(1, int((s >= s[0] + T * np.log(np.longdouble(min_p))).sum())))
    run = np.cumsum(w[:n])
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    i = min(int((run <= np.longdouble(u) * run[-1]).sum()), n - 1)
    return int(order[i]), float(z[i] - np.log(run[-1])), n
