"""Outputs laid over the queries with other strides are refused before any device work (no GPU needed)."""
import pytest

import paper_2608_08684_amd as rk
from test_paged_host import A, attention


@pytest.mark.parametrize("status, kw", [
    (A, dict(os_=264)), (A, dict(qs=512)), (A, dict(qs=512, os_=264)),
    (A, dict(sel={}, os_=512)), (A, dict(cache=dict(dtype=rk.RK_F32), os_=260)),
])
def test_outputs_over_the_queries_have_their_stride(status, kw):
    """A sequence's outputs would lie over another one's queries."""
    assert attention(**kw) == status and b"stride" in rk.load().rk_last_error()


def test_a_single_sequence_has_no_stride():
    """One row over another: only the workspace is wrong here."""
    assert attention(seqs=dict(n_seqs=1), os_=264, size=0) == rk.RK_ERR_WORKSPACE
