"""Paged attention where its workgroups outnumber the card's: the longest sequences go first, rows are split into two, three
and four parts, and pages are scored in a launch of their own."""
import numpy as np
import pytest

from paged_helpers import Case, check_attention
from test_gpu_paged_attention import check_selected

pytestmark = pytest.mark.gpu


def uneven(n, longest, seed):
    """Lengths with many equal ones, the longest last and empty sequences between."""
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(1, max(2, longest // 8), n)]
    for i in range(0, n, 5):
        lens[i] = 33
    for i in range(2, n, 9):
        lens[i] = 0
    lens[n // 2], lens[n - 1] = longest - 1, longest
    return lens


@pytest.mark.parametrize("n, heads, kv_heads, d, page, dtype, longest", [
    (64, 12, 12, 64, 16, "bf16", 500),      # 768 workgroups, a part a row
    (64, 32, 8, 128, 64, "bf16", 1000),     # exactly 512: in their order
    (64, 36, 9, 64, 16, "bf16", 900),       # 576
    (33, 8, 8, 64, 16, "bf16", 4300),       # four parts
    (33, 12, 12, 64, 32, "bf16", 4100),     # three
    (25, 24, 12, 64, 16, "bf16", 4000),     # two
    (64, 12, 12, 32, 16, "f32", 300),
    (33, 16, 8, 64, 16, "f32", 4300),
    (65, 12, 12, 64, 16, "bf16", 500),      # more sequences than a wave has lanes
])
def test_many_workgroups(n, heads, kv_heads, d, page, dtype, longest):
    import torch
    case = Case(uneven(n, longest, n), heads, kv_heads, d, page, dtype, seed=n + heads)
    # lengths that the call has to bound: negative ones, and ones past the table
    case.lengths[1], case.lengths[4], case.lengths[n - 2] = -3, -2 ** 31, 2 ** 31 - 1
    case.pages[n - 2] = case.pages[n - 1]
    ws = case.workspace()
    out, lse = case.outputs()
    case.cache.attention(case.seqs, case.q, out, ws, lse=lse)
    if longest % page:   # the row past the table sees what follows the last entry on its last page: NaN
        assert out[n - 2].isnan().all()
        case.lengths[n - 2] = longest
        case.cache.attention(case.seqs, case.q, out, ws, lse=lse)
    check_attention(case, out, lse)
    own = case.q.clone()
    case.cache.attention(case.seqs, own, own, ws)
    assert torch.equal(own, out)


def test_selected_with_scores_apart():
    """Four parts of a row for more workgroups than the card takes at a time: the pages are scored first."""
    lens = uneven(32, 17 * 256 - 5, 1)
    lens[3] = 16 * 256
    case = Case(lens, 16, 8, 64, 256, "bf16", seed=2, bounds=True)
    check_selected(case, 16, 1, 2)
