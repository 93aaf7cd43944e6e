"""Outputs laid over the queries with other strides, and calls of more workgroups than a launch takes, are refused before any
device work (no GPU needed)."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk
from test_paged_host import A, S, append, attention, logprobs


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


@pytest.mark.parametrize("cache, seqs, rows", [
    (dict(n_kv_heads=32, head_dim=128, dtype=rk.RK_F32), dict(n_seqs=1 << 23),
     dict(q=None, q_out=None, k_row_stride=4096, k_head_stride=128, v_row_stride=4096, v_head_stride=128)),
    (dict(), dict(n_seqs=1 << 23), dict()),
    (dict(n_kv_heads=65536), dict(n_seqs=1 << 14), dict(q=None, q_out=None)),
])
def test_appends_of_too_many_workgroups(cache, seqs, rows):
    assert append(cache=cache, seqs=seqs, rows=rows) == S and b"workgroups" in rk.load().rk_last_error()


def test_prompts_of_too_many_workgroups():
    offs = np.asarray([0, 1 << 30], np.int64)
    assert append(seqs=dict(n_seqs=1, max_pages=1 << 26, page_stride=1 << 26),
                  rows=dict(offsets=offs.ctypes.data, q=None, q_out=None)) == S
    assert b"workgroups" in rk.load().rk_last_error()


@pytest.mark.parametrize("rows, vocab", [(1 << 24, 10), ((1 << 24) + 1, 2), (1 << 24, 1 << 22), (1 << 22, 1 << 22)])
def test_log_probabilities_of_too_many_rows(rows, vocab):
    for dtype in (rk.RK_F32, rk.RK_BF16):
        if (rows, vocab, dtype) == (1 << 22, 1 << 22, rk.RK_BF16):
            rows *= 2
        assert logprobs(rows=rows, vocab=vocab, stride=vocab, dtype=dtype, size=1 << 60) == A
        assert b"n_rows" in rk.load().rk_last_error()
        assert rk.load().rk_token_logprobs_workspace_size(rows, vocab, dtype, 0) == 0


def test_log_probabilities_of_the_most_rows():
    assert rk.token_logprobs_workspace_size((1 << 24) - 1, 10) > 0
    assert logprobs(rows=(1 << 24) - 1, vocab=10, stride=10, size=0) == rk.RK_ERR_WORKSPACE
