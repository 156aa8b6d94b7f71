"""Plain CPU oracle of the layer-wise calls: rotation, page summaries, the choice of
pages, attention over them, adjusted logits and the choice over them.

TEST INFRASTRUCTURE ONLY (see pced_oracle). NumPy float64 and the plain definitions,
one row, page and token at a time; contiguous caches, no paging.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
SUM_EXP = 64  # summaries' scales are 2^-64 .. 2^64


def rotate(x: np.ndarray, pos: int, theta: float, rot: int, halves: bool) -> np.ndarray:
    """x [..., D]: pairs of the first `rot` dims turned by pos * theta^(-2j / rot)."""
    x = np.array(x, dtype=np.float64)
    y = x.copy()
    for j in range(rot // 2):
        a, b = (j, j + rot // 2) if halves else (2 * j, 2 * j + 1)
        ang = pos * theta ** (-2.0 * j / rot)
        c, s = math.cos(ang), math.sin(ang)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def _scale_exponent(top: float, rounded) -> int:
    """The smallest exponent e, within the limits, with rounded(top 2^-e) <= 127."""
    if not top > 0:
        return -SUM_EXP
    e = SUM_EXP if math.isinf(top) else min(max(math.frexp(top)[1] - 1 - 6, -SUM_EXP), SUM_EXP)
    while e < SUM_EXP and rounded(math.ldexp(top, -e)) > 127:
        e += 1
    return e


def summarize(k: np.ndarray):
    """Codes (max [D], min [D]) and exponent of one page's keys k [16][D]; NaN keys are left out."""
    k = np.asarray(k, dtype=np.float64)
    hi, lo = np.zeros(k.shape[1]), np.zeros(k.shape[1])
    for d in range(k.shape[1]):
        col = k[:, d][~np.isnan(k[:, d])]
        if col.size:
            hi[d], lo[d] = col.max(), col.min()
    e = _scale_exponent(float(np.maximum(np.abs(hi), np.abs(lo)).max()), math.ceil)
    clip = lambda x: np.clip(x, -127, 127).astype(np.int64)  # noqa: E731
    return clip(np.ceil(np.ldexp(hi, -e))), clip(np.floor(np.ldexp(lo, -e))), e


def query_weights(q: np.ndarray):
    """w+ [D], w- [D] as whole numbers, of a kv-head's q-heads q [G][D]."""
    q = np.asarray(q, dtype=np.float64)
    up, dn = np.where(q > 0, q, 0).sum(0), np.where(q < 0, q, 0).sum(0)
    e = _scale_exponent(float(max(up.max(), -dn.min())), lambda x: np.rint(x))
    return (np.clip(np.rint(np.ldexp(up, -e)), -127, 127).astype(np.int64),
            np.clip(np.rint(np.ldexp(dn, -e)), -127, 127).astype(np.int64))


def chosen_pages(q: np.ndarray, k: np.ndarray, n_pages: int, n_first: int, n_last: int) -> list:
    """Pages of a row and kv-head, ascending: q [G][D], k [tokens][D] (the row's own token last)."""
    pages = -(-len(k) // PAGE)
    if pages <= n_pages:
        return list(range(pages))
    up, dn = query_weights(q)
    found = []
    for p in range(n_first, pages - n_last):
        mx, mn, e = summarize(k[PAGE * p:PAGE * (p + 1)])
        found.append((-math.ldexp(int((up * mx).sum() + (dn * mn).sum()), e), p))
    found.sort()
    best = [p for _, p in found[:n_pages - n_first - n_last]]
    return sorted(list(range(n_first)) + best + list(range(pages - n_last, pages)))


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, pages) -> np.ndarray:
    """softmax(q k^T / sqrt(D)) v over the tokens of `pages`: q [G][D], k, v [tokens][D]."""
    at = [t for p in pages for t in range(PAGE * p, min(PAGE * (p + 1), len(k)))]
    s = np.asarray(q, np.float64) @ np.asarray(k, np.float64)[at].T / math.sqrt(q.shape[1])
    w = np.exp(s - s.max(axis=1, keepdims=True))
    return (w / w.sum(axis=1, keepdims=True)) @ np.asarray(v, np.float64)[at]


def adjust_row(s, history=(), repetition=1.0, presence=0.0, frequency=0.0, biases=(), allowed=None, real=np.float64):
    """Adjusted logits of one row [V]. history: tokens; biases: (token, value) in order, the last of a token
    counts; allowed: truth values [V] or None. real: the type that every operation rounds to."""
    s = np.array(s, dtype=real)
    V = len(s)
    count = {}
    for v in history:
        if 0 <= v < V:
            count[int(v)] = count.get(int(v), 0) + 1
    r, p, f = real(repetition), real(presence), real(frequency)
    with np.errstate(all="ignore"):
        for v, n in count.items():
            x = s[v] / r if s[v] > 0 else s[v] * r
            s[v] = (x - f * real(n)) - p
        for v, b in {int(v): b for v, b in biases if 0 <= v < V}.items():
            s[v] = s[v] + real(b)
    if allowed is not None:
        s[~np.asarray(allowed)] = -np.inf
    return s


def choose(rows, beta, prior, allowed=None, real=np.float64):
    """Eq. 2 and Eq. 3 over a query's adjusted rows [N + 1][V] (the amateur first): (token, expert, top1, top2),
    (-1, 0, -inf, -inf) where nothing can be chosen."""
    rows = np.asarray(rows, dtype=real)
    with np.errstate(all="ignore"):
        f = [((real(1) + real(b)) * rows[k + 1] - real(b) * rows[0]) + real(c) for k, (b, c) in enumerate(zip(beta, prior))]
    f = np.array(f)
    ok = ~np.isnan(f) & (f > -np.inf)
    if allowed is not None:
        ok &= np.asarray(allowed)[None, :]
    f = np.where(ok, f, -np.inf)
    S = f.max(axis=0)
    if not (S > -np.inf).any():
        return -1, 0, -np.inf, -np.inf
    y = int(np.argmax(S))
    rest = np.delete(S, y)
    return y, int(np.argmax(f[:, y])) + 1, float(S[y]), float(rest.max()) if rest.size else -np.inf
