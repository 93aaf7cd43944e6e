"""Paged caches of 8-bit values for the GPU tests."""
from __future__ import annotations

import numpy as np

from paged_helpers import Case


def rounded(x):
    """(codes float8_e4m3fn, scale bytes) of rows [..., d], from float64, by the format's definition (vectorised)."""
    import torch
    x = x.double().cpu()
    finite = torch.where(x.isfinite(), x, 0.0)
    m, e = torch.frexp(finite.abs().amax(-1))           # amax = m 2^e, 448 = 0.875 2^9
    e = (e.long() - 9 + (m > 0.875).long()).clamp(-117, 120)
    e = torch.where(m == 0, -117, e)
    unit = (e + 1023 << 52).view(torch.float64)[..., None]
    most = torch.where(e == 120, 240.0, 448.0)[..., None]
    y = torch.minimum(torch.maximum(finite / unit, -most), most)
    step = (torch.frexp(y.abs().clamp(min=2.0 ** -6))[1].long() - 4 + 1023 << 52).view(torch.float64)
    y = torch.where(x.isfinite(), torch.round(y / step) * step, float("nan"))
    return y.float().to(torch.float8_e4m3fn).cuda(), (e + 127).to(torch.uint8).cuda()


def values(codes, scales):
    """float64 values."""
    import torch
    return codes.float().double() * (scales.long() - 127 + 1023 << 52).view(torch.float64)[..., None]


class Case8(Case):
    """The same sequences in 8 bits; k and v are the bf16 numbers that the cache stands for.  What no sequence holds is
    NaN, with a scale byte of 255."""

    def __init__(self, lengths, heads, kv_heads, d, page, seed=0, bounds=False, **kw):
        import torch
        import paper_2608_08684_amd as rk
        super().__init__(lengths, heads, kv_heads, d, page, "bf16", seed=seed, **kw)
        unused = self.k[..., 0].isnan()
        self.raw = {}
        for name in "kv":
            x = getattr(self, name)
            # rows of very different size
            size = torch.randint(-12, 12, x.shape[:3], generator=torch.Generator().manual_seed(seed + 1)).cuda()
            x = x.float() * (torch.exp2(size.float())[..., None] if name == "v" else 1.0)
            codes, scales = rounded(torch.where(unused[..., None], 0.0, x))
            codes.view(torch.uint8)[unused] = 0x7F
            scales[unused] = 255
            self.raw[name], self.raw[name + "_scales"] = codes, scales
            setattr(self, name, torch.where(unused[..., None], float("nan"), values(codes, scales)).bfloat16())
        if bounds:
            x = self.k.float()
            lo = torch.where(x.isnan(), float("inf"), x).amin(2)
            hi = torch.where(x.isnan(), -float("inf"), x).amax(2)
            self.bounds = torch.stack([lo, hi], 2).bfloat16()
        self.plain = rk.PagedCache(self.k, self.v, self.bounds)
        self.cache = rk.PagedCache(self.raw["k"], self.raw["v"], self.bounds, k_scales=self.raw["k_scales"],
                                   v_scales=self.raw["v_scales"])


def empty_cache(n_pages, kv_heads, page, d, bounds=False):
    """(cache, its tensors): NaN everywhere, scale bytes 0."""
    import torch
    import paper_2608_08684_amd as rk
    k = torch.full((n_pages, kv_heads, page, d), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks = torch.zeros(n_pages, kv_heads, page, dtype=torch.uint8, device="cuda")
    b = torch.full((n_pages, kv_heads, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda") if bounds else None
    return rk.PagedCache(k, k.view(torch.uint8).clone().view(k.dtype), b, k_scales=ks, v_scales=ks.clone())
