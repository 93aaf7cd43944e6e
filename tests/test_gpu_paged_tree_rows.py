"""A drafted row's result is its own: no bit of it hangs on what the rows beside it score."""
import pytest

from test_gpu_paged_tree import Drafts, make
from tree_helpers import SHARED, lengths_of, shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form, dtype, d", [("narrow", "bf16", 64), ("narrow", "bf16", 128), ("narrow", "e4m3", 128),
                                            ("narrow", "f32", 32), ("narrow", "f32", 128)] +
                         [(form, dtype, d) for form in SHARED for dtype in ("bf16", "e4m3") for d in (64, 128)])
def test_rows_do_not_hang_on_each_other(form, dtype, d):
    """The other rows' queries eight times as large: their scores pass their references at many more tiles."""
    import torch
    if form == "narrow":
        case = make([3000, 700], 6, 2, d, 16, dtype, seed=5)
        drafts = Drafts(case, [5, 3], seed=5)
    else:
        case, drafts = shared(form, d, dtype, seed=5, lengths=[900] + lengths_of(form)[1:])
    mine = torch.arange(len(drafts.q), device="cuda") % 3 == 1
    ref, ref_lse = drafts.run()
    drafts.check(ref, ref_lse)
    drafts.q[~mine] *= 8
    out, lse = drafts.run()
    assert torch.equal(out[mine], ref[mine]) and torch.equal(lse[mine], ref_lse[mine])
    assert not torch.equal(out[~mine], ref[~mine])
