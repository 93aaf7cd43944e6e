"""Paged caches for the GPU tests: pages in any order, holes, and NaN wherever nothing was written."""
from __future__ import annotations

import numpy as np


def torch_dtype(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def half_step(name):
    """Half a rounding step of the type, relative to the value."""
    return 2.0 ** -8 if name == "bf16" else 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    """n sequences of the given lengths in pages dealt out at random; what no sequence holds is NaN."""

    def __init__(self, lengths, heads, kv_heads, d, page, dtype, seed=0, extra_pages=3, width=None, bounds=False):
        import torch
        import paper_2608_08684_amd as rk
        self.lens, self.H, self.G, self.d, self.page, self.dtype = list(lengths), heads, kv_heads, d, page, dtype
        g = torch.Generator().manual_seed(seed)
        n, count = len(lengths), [(max(x, 0) + page - 1) // page for x in lengths]
        width = width or max(max(count), 1)
        self.n_pages = sum(count) + extra_pages
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        table = torch.full((n, width), -1, dtype=torch.int32)
        k = torch.full((self.n_pages, kv_heads, page, d), float("nan"))
        v = torch.full((self.n_pages, kv_heads, page, d), float("nan"))
        at = 0
        for i, c in enumerate(count):
            table[i, :c] = order[at:at + c]
            for p in range(c):
                m = min(page, lengths[i] - p * page)
                k[order[at + p], :, :m] = torch.randn(kv_heads, m, d, generator=g)
                v[order[at + p], :, :m] = torch.randn(kv_heads, m, d, generator=g)
            at += c
        self.table = table
        self.k, self.v = k.to(torch_dtype(dtype)).cuda(), v.to(torch_dtype(dtype)).cuda()
        self.q = torch.randn(n, heads, d, generator=g).mul_(2.0).to(torch_dtype(dtype)).cuda()
        b = None
        if bounds:
            x = self.k.float()
            lo = torch.where(x.isnan(), float("inf"), x).amin(2)
            hi = torch.where(x.isnan(), -float("inf"), x).amax(2)
            b = torch.stack([lo, hi], 2).to(self.k.dtype)
        self.bounds = b
        self.pages, self.lengths = table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
        self.cache = rk.PagedCache(self.k, self.v, b)
        self.seqs = rk.PagedSeqs(self.pages, self.lengths)

    def workspace(self, select=0):
        import torch
        size = self.cache.workspace_size(len(self.lens), self.seqs.max_pages, self.H, select)
        assert size > 0
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN: nothing is taken from it unwritten

    def outputs(self):
        import torch
        n = len(self.lens)
        return (torch.full((n, self.H, self.d), float("nan"), dtype=self.k.dtype, device="cuda"),
                torch.full((n, self.H), float("nan"), device="cuda"))

    def rows(self, i, g, pages=None):
        """Keys and values of sequence i, KV head g (of the given pages of the sequence, or all)."""
        from oracle import paged as OP
        at = OP.entries(int(self.lengths[i]), self.pages[i].tolist(), self.page, self.n_pages)
        if pages is not None:
            keep = {int(self.pages[i, p]) for p in pages}
            at = [x for x in at if x[0] in keep]
        p, s = [x[0] for x in at], [x[1] for x in at]
        return f64(self.k[p, g, s]), f64(self.v[p, g, s])


def attention_tolerance(dtype, n, d, scale, out, weighted, products):
    """How far an output and its log-sum-exp may be off, from the roundings of one pass.

    A score is a sum of d fp32 products: off by at most (d + 8) 2^-24 of the summed |q k|, times the scale (delta).  A
    weight e^(s - m) then is off by a factor e^delta, its fp32 exponent and exponential by 2^-21 at these sizes, its
    two bf16 parts by 2^-16 (bf16 caches), so the output by twice that of the weighted |v|; sums run over n / 128 tiles
    of a wave, 64 within one and the joins: (n / 128 + 128) 2^-24.  The result is rounded once."""
    delta = (d + 8) * 2.0 ** -24 * products[:, None] * scale
    weight = 2 * (delta + 2.0 ** -21 + (2.0 ** -16 if dtype == "bf16" else 0.0)) + 2 * (n / 128 + 128) * 2.0 ** -24
    tol = half_step(dtype) * np.abs(out) * (1 + weight) + weight * weighted
    lse = delta[:, 0] + 2.0 ** -21 + (n / 128 + 128) * 2.0 ** -24
    return tol, lse


def check_attention(case, out, lse, scale=0.0, chosen=None):
    """Every output and log-sum-exp against float64; chosen[i][g]: the pages that were to be read."""
    from oracle import paged as OP
    scale = scale or 1.0 / np.sqrt(case.d)
    grp = case.H // case.G
    out, lse = f64(out), None if lse is None else f64(lse)
    q = f64(case.q)
    for i in range(len(case.lens)):
        for g in range(case.G):
            k, v = case.rows(i, g, None if chosen is None else chosen[i][g])
            h = slice(g * grp, (g + 1) * grp)
            o, l, weighted, products = OP.attend(q[i, h], k, v, scale)
            tol, ltol = attention_tolerance(case.dtype, len(k), case.d, scale, o, weighted, products)
            err = np.abs(out[i, h] - o)
            assert (err <= tol).all(), (i, g, len(k), float(err.max()), float(tol.flat[err.argmax()]))
            if lse is not None:
                if len(k) == 0:
                    assert (lse[i, h] == -np.inf).all() and not out[i, h].any()
                else:
                    assert (np.abs(lse[i, h] - l) <= ltol + 2.0 ** -22 * np.abs(l)).all(), (i, g)
