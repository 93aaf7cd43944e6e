"""Refusals of the paged-cache and log-probability calls, before any device work (no GPU needed)."""
import ctypes
import shutil
import subprocess
import os

import numpy as np
import pytest

import paper_2608_08684_amd as rk
from paper_2608_08684_amd import _PagedCache, _PagedRows, _PagedSeqs, _PageSelection

A, S, U, W = rk.RK_ERR_ARG, rk.RK_ERR_SHAPE, rk.RK_ERR_UNSUPPORTED, rk.RK_ERR_WORKSPACE
AT = 1 << 20    # an aligned address that is never read
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def make(cls, base, **kw):
    return cls(**{**base, **kw})


CACHE = dict(k=AT, v=AT, key_bounds=AT, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=rk.RK_BF16)
SEQS = dict(pages=AT, lengths=AT, page_stride=4, n_seqs=3, max_pages=4)
ROWS = dict(offsets=None, k=AT, v=AT, k_row_stride=128, k_head_stride=64, v_row_stride=128, v_head_stride=64, q=AT,
            q_out=AT, q_row_stride=256, q_out_row_stride=256, n_heads=4, rope_theta=1.0e4, positions=None)
CACHE_BAD = [
    (A, dict(k=None)), (A, dict(v=None)), (A, dict(k=AT + 8)), (A, dict(key_bounds=AT + 2)), (A, dict(n_pages=0)),
    (A, dict(n_pages=1 << 31)), (A, dict(n_kv_heads=0)), (A, dict(dtype=2)), (U, dict(page_size=8)),
    (U, dict(page_size=48)), (U, dict(page_size=512)), (U, dict(head_dim=32)), (U, dict(head_dim=96)),
    (U, dict(head_dim=256, dtype=rk.RK_F32)),
]
SEQS_BAD = [(A, dict(pages=None)), (A, dict(lengths=None)), (A, dict(n_seqs=0)), (A, dict(max_pages=0)),
            (A, dict(page_stride=3)), (S, dict(n_seqs=(1 << 23) + 1)),
            (S, dict(max_pages=(1 << 26) + 1, page_stride=1 << 27))]


def append(cache={}, seqs={}, rows={}):
    c, q, r = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs), make(_PagedRows, ROWS, **rows)
    return rk.load().rk_paged_append(ctypes.byref(c), ctypes.byref(q), ctypes.byref(r), None)


def attention(cache={}, seqs={}, sel=None, q=AT, qs=256, heads=4, scale=0.0, out=AT, os_=256, ws=AT, size=1 << 30):
    c, s = make(_PagedCache, CACHE, **cache), make(_PagedSeqs, SEQS, **seqs)
    if sel is None:
        return rk.load().rk_paged_attention(ctypes.byref(c), ctypes.byref(s), q, qs, heads, scale, out, os_, None, ws,
                                            size, None)
    p = make(_PageSelection, dict(n_select=4, keep_first=1, keep_last=1, selected=None), **sel)
    return rk.load().rk_paged_attention_selected(ctypes.byref(c), ctypes.byref(s), ctypes.byref(p), q, qs, heads,
                                                 scale, out, os_, None, ws, size, None)


@pytest.mark.parametrize("status, kw", CACHE_BAD)
def test_cache_refusals(status, kw):
    assert append(cache=kw) == status and rk.load().rk_last_error()
    assert attention(cache=kw) == status
    assert attention(cache=kw, sel={}) == status


@pytest.mark.parametrize("status, kw", SEQS_BAD)
def test_sequence_refusals(status, kw):
    assert append(seqs=kw) == status
    assert attention(seqs=kw) == status


def _offsets(*x):
    return np.asarray(x, np.int64)


@pytest.mark.parametrize("status, kw", [
    (A, dict(k=None)), (A, dict(v=None)), (A, dict(k=AT + 2)), (A, dict(v=AT + 8)), (A, dict(k_row_stride=132)),
    (A, dict(v_head_stride=68)), (A, dict(k_head_stride=-64)), (A, dict(k_row_stride=56)), (A, dict(v_head_stride=32)),
    (A, dict(q=None)), (A, dict(q_out=None)), (A, dict(n_heads=3)), (A, dict(n_heads=0)), (A, dict(q_row_stride=248)),
    (A, dict(q_out_row_stride=260)), (A, dict(q=AT + 4)), (A, dict(rope_theta=1.0)), (A, dict(rope_theta=-2.0)),
    (A, dict(rope_theta=float("nan"))), (A, dict(rope_theta=float("inf"))), (A, dict(q_out_row_stride=512)),
    (S, dict(offsets=_offsets(0, 2, 1, 3))), (S, dict(offsets=_offsets(1, 2, 3, 4))),
    (S, dict(offsets=_offsets(0, 1, 2, (1 << 30) + 1))),
])
def test_append_refusals(status, kw):
    if isinstance(kw.get("offsets"), np.ndarray):
        kw = dict(kw, offsets=kw["offsets"].ctypes.data)
    assert append(rows=kw) == status


def test_append_takes_a_batch_of_sequences_with_offsets():
    offs = np.arange(rk.RK_MAX_BATCH_SEQS + 2, dtype=np.int64)
    assert append(seqs=dict(n_seqs=rk.RK_MAX_BATCH_SEQS + 1), rows=dict(offsets=offs.ctypes.data)) == S


@pytest.mark.parametrize("status, kw", [
    (A, dict(q=None)), (A, dict(out=None)), (A, dict(ws=None)), (A, dict(ws=AT + 4)), (A, dict(q=AT + 2)),
    (A, dict(out=AT + 8)), (A, dict(qs=252)), (A, dict(qs=128)), (A, dict(os_=128)), (A, dict(heads=3)),
    (A, dict(heads=0)), (A, dict(scale=-1.0)), (A, dict(scale=float("nan"))), (A, dict(scale=float("inf"))),
    (W, dict(size=0)), (A, dict(sel=dict(n_select=0))), (A, dict(sel=dict(keep_first=-1))),
    (A, dict(sel=dict(keep_last=-1))), (A, dict(sel=dict(keep_first=2, keep_last=3))),
    (A, dict(sel=dict(keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1))), (A, dict(sel={}, cache=dict(key_bounds=None))),
    (S, dict(sel=dict(n_select=1 << 27))), (W, dict(sel={}, size=100)),
    (S, dict(seqs=dict(n_seqs=1 << 22))),
])
def test_attention_refusals(status, kw):
    assert attention(**kw) == status


def test_workspace_sizes():
    def size(n=3, pages=4, heads=4, select=0, **kw):
        c = make(_PagedCache, CACHE, **{**dict(k=None, v=None, key_bounds=None), **kw})
        return rk.load().rk_paged_workspace_size(ctypes.byref(c), n, pages, heads, select)
    assert size() > 0 and size(select=4) > size() and size(pages=4096) > size()
    # enough for fewer sequences and shorter tables, which may be split into more parts
    sizes = [[size(n=n, pages=p, heads=64, select=s) for n in (1, 2, 5, 31, 32, 64, 100, 127, 300, 640, 641, 1279, 4096)
              for p in (4, 8, 32, 64, 65, 100, 255, 256, 4096)] for s in (0, 1, 70, 300)]
    grids = [np.array(x, dtype=np.int64).reshape(13, 9) for x in sizes]
    for grid in grids:
        assert (np.diff(grid, axis=0) >= 0).all() and (np.diff(grid, axis=1) >= 0).all()
    assert all((b >= a).all() for a, b in zip(grids, grids[1:]))
    for bad in (dict(n=0), dict(pages=0), dict(heads=3), dict(select=-1), dict(page_size=20), dict(pages=1 << 27)):
        assert size(**bad) == 0
    sz = rk.token_logprobs_workspace_size
    assert sz(16, 10 ** 6, 5) > sz(16, 10 ** 6, 0) > sz(16, 32000, 5) > 0 and sz(1, 1 << 22, 32) > 0
    for vocab in (1000, 32000, 128256, 10 ** 6, 1 << 22):
        for dtype in ("f32", "bf16"):
            assert (np.diff([sz(n, vocab, 20, dtype) for n in (0, 1, 2, 3, 7, 16, 50, 64, 127, 128, 129, 256, 257, 2000)])
                    >= 0).all()
    assert sz(-1, 10, 0) == sz(1, 0, 0) == sz(1, 10, 11) == sz(1, 100, rk.RK_MAX_TOP + 1) == sz(1, 10, -1) == 0


def logprobs(logits=AT, dtype=rk.RK_F32, rows=2, vocab=100, stride=100, tokens=AT, n_top=0, lp=AT, rank=None,
             entropy=None, ids=None, top=None, ws=AT, size=1 << 20):
    return rk.load().rk_token_logprobs(logits, dtype, rows, vocab, stride, tokens, n_top, lp, rank, entropy, ids, top,
                                       ws, size, None)


@pytest.mark.parametrize("status, kw", [
    (A, dict(logits=None)), (A, dict(dtype=2)), (A, dict(rows=-1)), (A, dict(rows=1 << 25)), (A, dict(vocab=0)),
    (A, dict(vocab=(1 << 22) + 1, stride=1 << 23)),
    (A, dict(stride=99)), (A, dict(tokens=None)), (A, dict(tokens=None, lp=None, rank=AT)), (A, dict(lp=None)),
    (A, dict(n_top=-1, ids=AT)), (A, dict(n_top=33, ids=AT)), (A, dict(n_top=5)), (A, dict(ids=AT)),
    (A, dict(n_top=5, vocab=4, ids=AT)), (A, dict(ws=None)), (A, dict(ws=AT + 4)), (A, dict(logits=AT + 2)),
    (A, dict(logits=AT + 1, dtype=rk.RK_BF16)), (W, dict(size=16)),
])
def test_logprob_refusals(status, kw):
    assert logprobs(**kw) == status and rk.load().rk_last_error()


def test_no_rows_is_no_work():
    assert logprobs(rows=0) == rk.RK_OK
    offs = np.zeros(4, np.int64)
    assert append(rows=dict(offsets=offs.ctypes.data)) == rk.RK_OK


def test_host_tensors_are_refused():
    import torch
    k = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rk.PagedCache(k, k)
    with pytest.raises(ValueError):
        rk.PagedSeqs(torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        rk.token_logprobs(torch.zeros(1, 4), None, torch.zeros(256, dtype=torch.uint8), entropy=torch.zeros(1))


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    mirrors = {"rk_paged_cache": _PagedCache, "rk_paged_seqs": _PagedSeqs, "rk_paged_rows": _PagedRows,
               "rk_page_selection": _PageSelection}
    lines = []
    for name, cls in mirrors.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "rk.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0;\n}\n")
    exe = str(tmp_path / "layout")
    subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", exe], check=True)
    got = dict(l.split() for l in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, cls in mirrors.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)
