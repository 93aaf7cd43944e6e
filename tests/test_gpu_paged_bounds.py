"""Key bounds of pages with a Key that is not a number: it stays in its channels' bounds until the page starts again."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk

from paged_helpers import f64
from test_gpu_paged_append import Append

pytestmark = pytest.mark.gpu

SHAPES = [(4, 4, 64, 16, "bf16"), (8, 2, 128, 32, "bf16"), (2, 2, 32, 16, "f32"), (4, 2, 128, 64, "f32")]


def expected(a, before, filled):
    """Bounds over the stored Keys of the first filled[i] entries of each sequence; pages that hold none as before."""
    want, k = before.copy(), f64(a.k)
    for i, n in enumerate(filled):
        for p in range((n + a.page - 1) // a.page):
            rows = k[int(a.pages[i, p]), :, :min(a.page, n - p * a.page)]
            want[int(a.pages[i, p]), :, 0], want[int(a.pages[i, p]), :, 1] = rows.min(1), rows.max(1)
    return want


def same(x, y):
    return np.array_equal(x, y, equal_nan=True)


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("theta", [0.0, 1.0e4])
def test_nan_keys_stay_in_the_bounds(heads, kv_heads, d, page, dtype, theta):
    total = 3 * page + 5
    for step in (total, page, 7, 1):
        a = Append([total, total], [total, total], heads, kv_heads, d, page, dtype, seed=step, theta=theta, queries=False)
        a.new_k[0, 0, 3] = float("nan")                     # the first entry of a page
        a.new_k[page + 9, kv_heads - 1, d - 1] = float("nan")
        a.new_k[total + 2 * page - 1, 0, 0] = float("nan")  # the last one
        before = f64(a.bounds)
        cache, seqs = rk.PagedCache(a.k, a.v, a.bounds), rk.PagedSeqs(a.pages, a.lengths)
        for r in range(0, total, step):
            m = min(step, total - r)
            a.lengths.fill_(r + m)
            rows = [x for s in (0, total) for x in range(s + r, s + r + m)]
            cache.append(seqs, a.new_k[rows], a.new_v[rows], row_offsets=[0, m, 2 * m], rope_theta=theta)
            got = f64(a.bounds)
            assert same(got, expected(a, before, [r + m] * 2)), (step, r)
        assert np.isnan(got).any() and np.isfinite(got).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_page_that_starts_again_forgets(dtype):
    a = Append([20], [20], 2, 2, 64, 16, dtype, seed=1, theta=0.0, queries=False)
    a.new_k[4] = float("nan")
    a.call()
    assert np.isnan(f64(a.bounds)[int(a.pages[0, 0])]).all() and np.isfinite(f64(a.bounds)[int(a.pages[0, 1])]).all()
    a.new_k[4] = 1.0
    before = f64(a.bounds)
    a.call()
    assert same(f64(a.bounds), expected(a, before, [20])) and np.isfinite(f64(a.bounds)).all()


def test_pages_with_nan_bounds_are_chosen_last():
    """A score that is not a number counts as -inf; the pages that are always kept are kept all the same."""
    import torch
    a = Append([160], [160], 2, 1, 64, 16, "f32", seed=2, theta=0.0, queries=False)
    a.new_k[[16 * 3 + 1, 16 * 7], 0, 5] = float("nan")
    a.call()
    cache, seqs = rk.PagedCache(a.k, a.v, a.bounds), rk.PagedSeqs(a.pages, a.lengths)
    q = torch.ones(1, 2, 64, device="cuda")
    ws = torch.empty(cache.workspace_size(1, 10, 2, 9), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for n, want in ((8, [0, 1, 2, 4, 5, 6, 8, 9]), (9, [0, 1, 2, 3, 4, 5, 6, 8, 9])):
        sel = torch.empty(1, 1, n, dtype=torch.int32, device="cuda")
        cache.attention_selected(seqs, q, out, ws, n_select=n, keep_first=1, keep_last=1, selected=sel)
        assert sel[0, 0].tolist() == want and out.isnan().any() == (3 in want)
