"""Paged key-value cache, token log probabilities and beams in float64, position by position.

Written from the definitions of ``include/rk.h``; shares nothing with the library.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["rotate", "entries", "append_rows", "attend", "page_scores", "choose_pages", "logprobs", "e4m3", "visible",
           "kept_moves", "reordered", "beam_select"]


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


def _round_e4m3(y):
    """The nearest of the 8-bit values, ties to the even one; |y| at most 448."""
    if y == 0 or y != y:
        return y
    step = 2.0 ** (max(math.frexp(y)[1], -5) - 4)      # 4 significant bits, whole steps of 2^-9 below 2^-6
    return round(y / step) * step                        # Python rounds halves to even


def e4m3(row):
    """(values in units of the scale, scale byte) of one row: the least power of two, 2^-117 at least, of which the
    largest finite magnitude is at most 448; infinities and NaN are NaN, what would round to 2^128 stays below."""
    row = np.asarray(row, np.float64)
    finite = np.isfinite(row)
    top = float(np.abs(row[finite]).max()) if finite.any() else 0.0
    e = -117
    while top > 448.0 * 2.0 ** e:
        e += 1
    most = 240.0 if e == 120 else 448.0
    return [_round_e4m3(min(max(x / 2.0 ** e, -most), most)) if f else math.nan for x, f in zip(row, finite)], e + 127


def visible(length, m, mask, n_entries):
    """Entries (below n_entries) that a draft of the last m sees; mask None: all."""
    b = int(length) - m
    return [u for u in range(max(0, min(int(length), n_entries))) if u < b or mask is None or mask >> (u - b) & 1]


def kept_moves(length, m, kept):
    """(new entry, old entry) of the path of a sequence's drafts."""
    b, moves, last = int(length) - m, [], -1
    for j, t in enumerate(kept):
        if not last < t < m:
            break
        moves.append((b + j, b + int(t)))
        last = t
    return moves


def reordered(pages, lengths, parents, n_beams, page_size):
    """(new table, [(page, source page, entries)]) of the sequences after a selection."""
    new, copies = [list(map(int, row)) for row in pages], []
    for i, p in enumerate(parents):
        first = i // n_beams * n_beams
        src = first + p if 0 <= p < n_beams else i
        length = max(0, min(int(lengths[first]), len(pages[i]) * page_size))
        full, rest = length // page_size, length % page_size
        new[i][:full] = [int(x) for x in pages[src][:full]]
        if rest and src != i:
            copies.append((int(pages[i][full]), int(pages[src][full]), rest))
    return new, copies


def beam_select(logits, scores, ended, end_token, n_out):
    """(parent, token, score) of the n_out best candidates of a group's beams."""
    found = []
    for b, (x, s) in enumerate(zip(logits, scores)):
        if not s > -math.inf:
            continue
        if ended is not None and ended[b]:
            found.append((-float(s), b, 0.0, end_token))
            continue
        x = np.asarray(x, np.float64)
        m = x.max() if not np.isnan(x).any() else math.nan
        if not math.isfinite(m):
            continue
        logp = (x - m) - math.log(np.sum(np.exp(x - m)))
        best = [int(v) for v in np.argsort(-x, kind="stable")[:n_out]]
        found += [(-(float(s) + logp[v]), b, -x[v], v) for v in best if x[v] > -math.inf]
    found = sorted(found)[:n_out]
    return [(b, v, -s) for s, b, _, v in found] + [(-1, -1, -math.inf)] * (n_out - len(found))
