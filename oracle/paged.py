"""Paged key-value cache and token log probabilities in float64, position by position.

Written from the definitions of ``include/rk.h``; shares nothing with the library.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["rotate", "entries", "append_rows", "attend", "page_scores", "choose_pages", "logprobs"]


def rotate(x, position, theta):
    """Rotate-half rotary embedding of x [heads, d] at one position; theta 0: none."""
    x = np.asarray(x, np.float64)
    if theta == 0:
        return x.copy()
    half = x.shape[-1] // 2
    a = position * np.asarray([theta ** (-2.0 * j / x.shape[-1]) for j in range(half)])
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def entries(length, pages, page_size, n_pages):
    """(page, slot) of each entry that a sequence can see, in order; pages outside the cache hold nothing."""
    length = max(0, min(int(length), len(pages) * page_size))
    return [(int(pages[e // page_size]), e % page_size) for e in range(length)
            if 0 <= pages[e // page_size] < n_pages]


def append_rows(lengths, counts, pages, page_size, n_pages):
    """(row, page, slot) of each new row that is written, and (row, entry) of every new row."""
    written, every, row = [], [], 0
    for length, m, table in zip(lengths, counts, pages):
        for j in range(m):
            e = int(length) - m + j
            every.append((row, e))
            if 0 <= e < len(table) * page_size and 0 <= table[e // page_size] < n_pages:
                written.append((row, int(table[e // page_size]), e % page_size))
            row += 1
    return written, every


def attend(q, k, v, scale):
    """q [heads, d] over k, v [n, d]: outputs, log-sum-exps, weights times |v|, and the largest sum of |q k|."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros_like(q), np.full(len(q), -np.inf), np.zeros_like(q), np.zeros(len(q))
    s = scale * (q @ k.T)
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    total = p.sum(1, keepdims=True)
    p /= total
    return p @ v, (m + np.log(total))[:, 0], p @ np.abs(v), (np.abs(q) @ np.abs(k).T).max(1)


def page_scores(q, bounds):
    """Sum over the heads q [heads, d] and channels of max(q lo, q hi), 0 where q is; bounds [pages, 2, d]."""
    q, b = np.asarray(q, np.float64), np.asarray(bounds, np.float64)
    scores = []
    for lo, hi in b:
        with np.errstate(invalid="ignore"):
            terms = np.where(q == 0, 0.0, np.maximum(q * lo, q * hi)).ravel()
        scores.append(math.fsum(terms) if np.isfinite(terms).all() else float(np.sum(terms)))
    return np.asarray(scores)


def choose_pages(scores, valid, n_select, keep_first, keep_last):
    """The pages (increasing) that a query reads."""
    n = len(scores)
    key = [(-math.inf if p < keep_first or p >= n - keep_last else -(scores[p] if scores[p] == scores[p] else -math.inf), p)
           for p in range(n) if valid[p]]
    return sorted(p for _, p in sorted(key)[:n_select])


def logprobs(x, token, n_top):
    """logprob, rank, entropy, top ids and top logprobs of one row of logits."""
    x = np.asarray(x, np.float64)
    order = sorted(range(len(x)), key=lambda i: (-(x[i] if x[i] == x[i] else -math.inf), i))
    m = x[order[0]]
    if not math.isfinite(m) or np.isnan(x).any():
        logp = np.full(len(x), np.nan)
        entropy = math.nan
    else:
        logp = (x - m) - math.log(math.fsum(np.exp(x - m)))
        seen = logp > -np.inf
        entropy = -math.fsum(np.exp(logp[seen]) * logp[seen])
    has = token is not None and 0 <= token < len(x)
    return (logp[token] if has else 0.0, 1 + order.index(token) if has else 0, entropy, order[:n_top],
            logp[order[:n_top]])
