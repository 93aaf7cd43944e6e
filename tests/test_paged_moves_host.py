"""Refusals of the 8-bit caches, reads, drafts and beams, before any device work (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2608_08684_amd as rk
from paper_2608_08684_amd import _PagedCache, _PagedSeqs

from test_paged_host import A, AT, CACHE, CACHE_BAD, S, SEQS, SEQS_BAD, U, W, append, attention, make

E4M3 = dict(dtype=rk.RK_E4M3, k_scales=AT, v_scales=AT)


def _at(offsets):
    return offsets.ctypes.data if offsets is not None else None


def _offsets(*x):
    return np.asarray(x, np.int64)


def read(cache={}, seqs={}, offsets=None, k=AT, krs=128, khs=64, v=AT, vrs=128, vhs=64):
    c, q = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs)
    return rk.load().rk_paged_read(ctypes.byref(c), ctypes.byref(q), _at(offsets), k, krs, khs, v, vrs, vhs, None)


def tree(cache={}, seqs={}, offsets=_offsets(0, 1, 5, 5), masks=AT, q=AT, qs=256, heads=4, scale=0.0, out=AT, os_=256,
         ws=AT, size=1 << 30):
    c, s = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs)
    return rk.load().rk_paged_attention_tree(ctypes.byref(c), ctypes.byref(s), _at(offsets), masks, q, qs, heads, scale,
                                             out, os_, None, ws, size, None)


def keep(cache={}, seqs={}, offsets=_offsets(0, 1, 5, 5), kept=AT, stride=8, n_kept=8):
    c, s = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs)
    return rk.load().rk_paged_keep(ctypes.byref(c), ctypes.byref(s), _at(offsets), kept, stride, n_kept, None)


def reorder(cache={}, seqs={}, beams=3, parents=AT, out=AT + 4096, stride=4):
    c, s = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs)
    return rk.load().rk_paged_reorder(ctypes.byref(c), ctypes.byref(s), beams, parents, out, stride, None)


CALLS = (read, tree, keep, reorder)


@pytest.mark.parametrize("status, kw", CACHE_BAD)
def test_cache_refusals(status, kw):
    assert all(call(cache=kw) == status and rk.load().rk_last_error() for call in CALLS)


@pytest.mark.parametrize("status, kw", SEQS_BAD)
def test_sequence_refusals(status, kw):
    assert all(call(seqs=kw) == status for call in CALLS)


@pytest.mark.parametrize("status, kw", [
    (A, dict(k_scales=None)), (A, dict(v_scales=None)), (A, dict(k_scales=AT + 1)), (A, dict(v_scales=AT + 8)),
    (U, dict(head_dim=32)), (U, dict(head_dim=96)), (A, dict(k=AT + 8)),
])
def test_e4m3_cache_refusals(status, kw):
    bad = {**E4M3, **kw}
    assert append(cache=bad) == status and attention(cache=bad) == status and attention(cache=bad, sel={}) == status
    assert all(call(cache=bad) == status for call in CALLS)


def test_e4m3_rows_are_bf16():
    """Strides count bf16 elements: 8 are a 16-byte piece."""
    assert append(cache=E4M3, rows=dict(k_row_stride=132)) == A and attention(cache=E4M3, qs=260) == A
    assert read(cache=E4M3, krs=132) == A and tree(cache=E4M3, qs=260) == A
    c = make(_PagedCache, CACHE, k=None, v=None, key_bounds=None, dtype=rk.RK_E4M3)
    bf = make(_PagedCache, CACHE, k=None, v=None, key_bounds=None)
    size = rk.load().rk_paged_workspace_size
    assert size(ctypes.byref(c), 3, 4096, 4, 5) == size(ctypes.byref(bf), 3, 4096, 4, 5) > 0


def test_e4m3_is_for_caches_only():
    assert rk.load().rk_token_logprobs(AT, rk.RK_E4M3, 2, 100, 100, AT, 0, AT, None, None, None, None, AT, 1 << 20,
                                       None) == A


@pytest.mark.parametrize("status, kw", [
    (A, dict(k=None, v=None)), (A, dict(k=AT + 2)), (A, dict(v=AT + 8)), (A, dict(krs=132)), (A, dict(vhs=68)),
    (A, dict(khs=-64)), (A, dict(krs=56)), (A, dict(vhs=32)), (S, dict(offsets=_offsets(0, 2, 1, 3))),
    (S, dict(offsets=_offsets(1, 2, 3, 4))), (S, dict(offsets=_offsets(0, 1, 2, (1 << 30) + 1))),
    (S, dict(offsets=_offsets(0, 1, 2, 1 << 30))),
])
def test_read_refusals(status, kw):
    assert read(**kw) == status


@pytest.mark.parametrize("status, kw", [
    (A, dict(offsets=None)), (S, dict(offsets=_offsets(0, 2, 1, 3))), (S, dict(offsets=_offsets(1, 2, 3, 4))),
    (S, dict(offsets=_offsets(0, 1, 2, 67))), (A, dict(q=None)), (A, dict(out=None)), (A, dict(ws=None)),
    (A, dict(ws=AT + 4)), (A, dict(masks=AT + 4)), (A, dict(q=AT + 2)), (A, dict(out=AT + 8)), (A, dict(qs=252)),
    (A, dict(qs=128)), (A, dict(os_=128)), (A, dict(os_=264)), (A, dict(heads=3)), (A, dict(heads=0)),
    (A, dict(scale=-1.0)), (A, dict(scale=float("nan"))), (A, dict(scale=float("inf"))), (W, dict(size=0)),
    (S, dict(heads=1 << 23, qs=1 << 30, os_=1 << 30)),
])
def test_tree_refusals(status, kw):
    assert tree(**kw) == status and rk.load().rk_last_error()


def test_at_most_a_batch_of_sequences_with_drafts():
    n = rk.RK_MAX_BATCH_SEQS + 1
    offs = np.arange(n + 1, dtype=np.int64)
    assert tree(seqs=dict(n_seqs=n), offsets=offs) == S and keep(seqs=dict(n_seqs=n), offsets=offs) == S
    assert read(seqs=dict(n_seqs=n), offsets=offs) == S


@pytest.mark.parametrize("status, kw", [
    (A, dict(offsets=None)), (A, dict(kept=None)), (A, dict(n_kept=0)), (A, dict(n_kept=65, stride=65)),
    (A, dict(stride=7)), (S, dict(offsets=_offsets(0, 2, 1, 3))), (S, dict(offsets=_offsets(0, 1, 2, 67))),
])
def test_keep_refusals(status, kw):
    assert keep(**kw) == status


@pytest.mark.parametrize("status, kw", [
    (A, dict(parents=None)), (A, dict(beams=0)), (A, dict(beams=2)), (A, dict(beams=33, seqs=dict(n_seqs=33))),
    (A, dict(stride=3)), (A, dict(out=AT, stride=5)), (S, dict(seqs=dict(n_seqs=3 << 21), cache=dict(n_kv_heads=100))),
])
def test_reorder_refusals(status, kw):
    assert reorder(**kw) == status


def test_no_rows_are_no_work():
    none = np.zeros(4, np.int64)
    assert read(offsets=none) == tree(offsets=none, q=None, out=None, ws=None) == keep(offsets=none) == rk.RK_OK


def select(logits=AT, dtype=rk.RK_F32, groups=2, beams=3, vocab=100, stride=100, scores=AT, ended=None, n_out=3,
           parents=AT, tokens=AT, out=AT + 4096, ws=AT, size=1 << 20):
    return rk.load().rk_beam_select(logits, dtype, groups, beams, vocab, stride, scores, ended, -1, n_out, parents,
                                    tokens, out, ws, size, None)


@pytest.mark.parametrize("status, kw", [
    (A, dict(logits=None)), (A, dict(dtype=rk.RK_E4M3)), (A, dict(dtype=3)), (A, dict(groups=-1)), (A, dict(beams=0)),
    (A, dict(beams=33)), (A, dict(vocab=0)), (A, dict(vocab=(1 << 22) + 1, stride=1 << 23)), (A, dict(stride=99)),
    (A, dict(scores=None)), (A, dict(n_out=0)), (A, dict(n_out=33)), (A, dict(parents=None)), (A, dict(tokens=None)),
    (A, dict(out=None)), (A, dict(ws=None)), (A, dict(ws=AT + 4)), (A, dict(logits=AT + 2)),
    (A, dict(logits=AT + 1, dtype=rk.RK_BF16)), (A, dict(out=AT, n_out=4)), (W, dict(size=16)),
    (A, dict(groups=1 << 24)),
])
def test_beam_select_refusals(status, kw):
    assert select(**kw) == status and rk.load().rk_last_error()


def test_no_groups_are_no_work():
    assert select(groups=0, logits=None, scores=None) == rk.RK_OK


def test_workspace_sizes():
    def size(n=3, rows=40, pages=64, heads=4, **kw):
        c = make(_PagedCache, CACHE, **{**dict(k=None, v=None, key_bounds=None), **kw})
        return rk.load().rk_paged_tree_workspace_size(ctypes.byref(c), n, rows, pages, heads)
    # enough for fewer sequences and rows, and shorter tables
    grid = np.array([[[size(n=n, rows=r, pages=p) for p in (1, 16, 33, 64, 500, 4096)] for r in (1, 5, 17, 40, 64)]
                     for n in (1, 2, 7, 64)], dtype=np.int64)
    assert (grid > 0).all() and all((np.diff(grid, axis=i) >= 0).all() for i in range(3)) and grid.max() > 256
    for bad in (dict(n=0), dict(n=65), dict(pages=0), dict(rows=-1), dict(rows=193), dict(heads=3), dict(page_size=20),
                dict(pages=1 << 27)):
        assert size(**bad) == 0
    sz = rk.beam_select_workspace_size
    for vocab in (1, 20, 1000, 50257, 128256, 1 << 22):
        for dtype in ("f32", "bf16"):
            for n_out in (1, 8, 32):
                sizes = [sz(g, 4, vocab, n_out, dtype) for g in (0, 1, 2, 3, 16, 17, 32, 64, 65, 300)]
                assert sizes[0] > 0 and (np.diff(sizes) >= 0).all()
    assert sz(-1, 4, 10, 1) == sz(1, 0, 10, 1) == sz(1, 33, 10, 1) == sz(1, 4, 10, 33) == sz(1, 4, 10, 0) == 0


def test_host_tensors_are_refused():
    import torch
    k = torch.zeros(2, 2, 16, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 2, 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        rk.PagedCache(k, k, k_scales=s, v_scales=s)
    f, i = torch.zeros(1, 1), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        rk.beam_select(torch.zeros(1, 4), f, i, i, f, torch.zeros(256, dtype=torch.uint8))
