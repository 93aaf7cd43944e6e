"""Attention of one new token over a paged cache, whole and over selected pages, against float64.

Whatever no sequence holds - the rest of a last page, free pages, pages that a table names wrongly - is NaN, and so is
the workspace before the call."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk
from oracle import paged as OP

from gpu_helpers import log
from paged_helpers import Case, check_attention, f64, torch_dtype

pytestmark = pytest.mark.gpu

EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
SHAPES = [  # heads, KV heads, head size, page, dtype
    (4, 4, 64, 16, "bf16"), (8, 2, 128, 16, "bf16"), (6, 2, 128, 64, "bf16"), (16, 1, 64, 256, "bf16"),
    (20, 1, 128, 32, "bf16"), (35, 1, 64, 16, "bf16"), (2, 2, 32, 16, "f32"), (4, 4, 64, 16, "f32"),
    (8, 2, 128, 32, "f32"), (17, 1, 128, 128, "f32"), (12, 12, 64, 128, "bf16"),
]


def attend(case, **kw):
    out, lse = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace(), lse=lse, **kw)
    return out, lse


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
def test_short_lengths(heads, kv_heads, d, page, dtype):
    case = Case(EDGES, heads, kv_heads, d, page, dtype, seed=heads)
    check_attention(case, *attend(case))


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
def test_long_lengths_are_split_and_joined(heads, kv_heads, d, page, dtype):
    case = Case([5000, 0, 1, 257, 4096, 3001], heads, kv_heads, d, page, dtype, seed=1)
    check_attention(case, *attend(case))


def test_one_long_sequence():
    case = Case([33333], 8, 2, 128, 16, "bf16", seed=2)
    check_attention(case, *attend(case))


def test_many_sequences():
    case = Case([(7 * i) % 91 for i in range(300)], 4, 4, 64, 16, "bf16", seed=3)
    check_attention(case, *attend(case))


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 32)])
@pytest.mark.parametrize("scale", [0.0, 0.01, 1.0])
def test_scale_and_no_lse(dtype, d, scale):
    case = Case([300, 40], 4, 2, d, 16, dtype, seed=4)
    out, _ = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace(), scale=scale)
    check_attention(case, out, None, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 37, 255, 256, 1029])
def test_one_key_decides(dtype, at):
    """A key with a far larger product than all others takes the whole weight, wherever it lies."""
    import torch
    case = Case([1030], 4, 2, 64, 16, dtype, seed=5)
    page, slot = int(case.table[0, at // 16]), at % 16
    case.k[page, :, slot] = 40.0 * case.q[0].view(2, 2, 64)[:, 0] / case.q[0].view(2, 2, 64)[:, 0].float().norm(
        dim=-1, keepdim=True).to(case.q.dtype)
    out, lse = attend(case)
    check_attention(case, out, lse)
    assert torch.equal(out[0, 0::2], case.v[page, :, slot])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tables_with_holes_and_wrong_pages(dtype):
    """Ids outside the cache hold nothing; a sequence that has only such pages sees nothing."""
    case = Case([100, 500, 64, 900, 33], 4, 2, 64, 16, dtype, seed=6)
    for i, p, bad in ((0, 0, -1), (0, 6, case.n_pages), (1, 3, 2 ** 31 - 1), (1, 4, -2 ** 31), (3, 56, -7)):
        case.pages[i, p] = bad
    case.pages[2, :] = -1
    check_attention(case, *attend(case))


def test_lengths_outside_the_table():
    """Negative lengths are empty; lengths past the table are those of the table."""
    import torch
    case = Case([64, 64, 64], 4, 2, 64, 16, "bf16", seed=7, width=4)
    case.lengths.copy_(torch.tensor([-5, 1000, 2 ** 31 - 1], dtype=torch.int32))
    check_attention(case, *attend(case))


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 64)])
def test_strides(dtype, d):
    """Queries as columns of a wider row, outputs into one, tables with longer rows."""
    import torch
    case = Case([77, 300, 1], 4, 2, d, 16, dtype, seed=8)
    t = torch_dtype(dtype)
    wide_q = torch.full((3, 4 * d + 64), float("nan"), dtype=t, device="cuda")
    wide_q[:, 32:32 + 4 * d] = case.q.view(3, -1)
    wide_o = torch.full((3, 4 * d + 16), -7.0, dtype=t, device="cuda")
    pages = torch.full((3, case.pages.shape[1] + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    pages[:, :case.pages.shape[1]] = case.pages
    seqs = rk.PagedSeqs(pages[:, :case.pages.shape[1]], case.lengths)
    _, lse = case.outputs()
    case.cache.attention(seqs, wide_q[:, 32:32 + 4 * d].view(3, 4, d), wide_o[:, :4 * d].view(3, 4, d),
                         case.workspace(), lse=lse)
    check_attention(case, wide_o[:, :4 * d].reshape(3, 4, d), lse)
    assert (wide_o[:, 4 * d:] == -7.0).all()


def test_non_finite_values_stay_with_their_sequence():
    """An infinity or NaN that a sequence holds reaches its own outputs, and nothing else's."""
    case = Case([50, 50, 50], 4, 2, 64, 16, "bf16", seed=9)
    ref, _ = attend(case)
    case.v[int(case.table[1, 1]), 0, 3, 7] = float("inf")
    case.k[int(case.table[2, 0]), 1, 2, 5] = float("nan")
    out, _ = attend(case)
    assert (out[0] == ref[0]).all() and (out[1, 2:] == ref[1, 2:]).all() and (out[2, :2] == ref[2, :2]).all()
    assert out[1, :2, 7].isinf().all() and out[2, 2:].isnan().all()
    keep = [x for x in range(64) if x != 7]
    assert (out[1, :2][:, keep] == ref[1, :2][:, keep]).all()


def test_a_cache_beyond_32_bit_offsets():
    """Pages whose byte offsets need more than 32 bits."""
    import torch
    G, d, page = 8, 128, 256
    n_pages = 5 * 2 ** 30 // (G * page * d * 2)     # 5 GiB of keys, and of values
    k = torch.empty(n_pages, G, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Case([700], 16, G, d, page, "bf16", seed=10, extra_pages=0)
    at = [n_pages - 1, n_pages // 2, n_pages - 3]
    for p, far in enumerate(at):
        k[far], v[far] = small.k[int(small.table[0, p])], small.v[int(small.table[0, p])]
    cache = rk.PagedCache(k, v)
    seqs = rk.PagedSeqs(torch.tensor([at], dtype=torch.int32, device="cuda"), small.lengths)
    out, lse = small.outputs()
    cache.attention(seqs, small.q, out, small.workspace(), lse=lse)
    ref, ref_lse = attend(small)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    check_attention(small, out, lse)


# ----------------------------------------------------------------------------- selected pages

def choose(case, n_select, first, last):
    q, b, grp = f64(case.q), f64(case.bounds), case.H // case.G
    chosen = []
    for i in range(len(case.lens)):
        length = max(0, min(int(case.lengths[i]), case.pages.shape[1] * case.page))
        count = (length + case.page - 1) // case.page
        row = case.pages[i, :count].tolist()
        valid = [0 <= p < case.n_pages for p in row]
        at = [p if ok else 0 for p, ok in zip(row, valid)]
        chosen.append([OP.choose_pages(OP.page_scores(q[i, g * grp:(g + 1) * grp], b[at, g]) if count else [], valid,
                                       n_select, first, last) for g in range(case.G)])
    return chosen


def run_selected(case, n_select, first, last):
    import torch
    out, lse = case.outputs()
    sel = torch.full((len(case.lens), case.G, n_select), -9, dtype=torch.int32, device="cuda")
    case.cache.attention_selected(case.seqs, case.q, out, case.workspace(n_select), n_select=n_select,
                                  keep_first=first, keep_last=last, lse=lse, selected=sel)
    return out, lse, sel


def check_selected(case, n_select, first, last):
    out, lse, sel = run_selected(case, n_select, first, last)
    chosen = choose(case, n_select, first, last)
    sel = sel.cpu().numpy()
    for i, row in enumerate(chosen):
        for g, want in enumerate(row):
            assert sel[i, g].tolist() == want + [-1] * (n_select - len(want)), (i, g)
    check_attention(case, out, lse, chosen=chosen)


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("n_select, first, last", [(1, 0, 0), (4, 1, 2), (9, 0, 1), (40, 3, 3)])
def test_selected_pages(heads, kv_heads, d, page, dtype, n_select, first, last):
    case = Case([0, 1, page, page + 1, 6 * page + 5, 23 * page, 61 * page - 3], heads, kv_heads, d, page, dtype,
                seed=heads + n_select, bounds=True)
    check_selected(case, n_select, first, last)


def test_selected_long():
    case = Case([40000, 12345], 8, 2, 64, 16, "bf16", seed=11, bounds=True)
    check_selected(case, 250, 1, 4)


def test_more_pages_than_the_sequences_have():
    case = Case([100, 17], 4, 2, 64, 16, "f32", seed=12, bounds=True)
    check_selected(case, 64, 2, 2)


@pytest.mark.parametrize("n_select", [3, 1023, 1024, 1025])
@pytest.mark.parametrize("pages", [1, 1023, 1024, 1025])
def test_around_a_thousand_pages(pages, n_select):
    case = Case([16 * pages - 5, 16 * (pages // 2)], 2, 1, 64, 16, "bf16", seed=pages + n_select, bounds=True)
    check_selected(case, n_select, 0, 2)


def test_ties_go_to_the_lower_page():
    """Pages with the same bounds, and a query of zeros (every score 0)."""
    case = Case([640, 640], 4, 2, 64, 16, "bf16", seed=13, bounds=True)
    case.bounds[case.pages[0].long()] = case.bounds[int(case.pages[0, 0])].clone()
    case.q[1] = 0
    check_selected(case, 7, 0, 1)
    *_, sel = run_selected(case, 7, 0, 1)
    assert (sel.cpu() == sel.new_tensor([0, 1, 2, 3, 4, 5, 39]).cpu()).all()


def test_signed_zeros_are_one_score():
    case = Case([160], 1, 1, 64, 16, "f32", seed=14, bounds=True)
    case.bounds.zero_()
    case.bounds[case.pages[0, ::2].long()] = -0.0
    check_selected(case, 4, 0, 0)


def test_selection_passes_over_what_holds_nothing():
    """Wrong page ids are never chosen, not even where pages are always kept; too few pages leave -1."""
    case = Case([320, 320, 160], 4, 2, 64, 16, "bf16", seed=15, bounds=True)
    for i, p in ((0, 0), (0, 7), (0, 19), (1, 19)):
        case.pages[i, p] = -1 if p else case.n_pages
    case.pages[2, :] = -1
    check_selected(case, 19, 1, 1)
    check_selected(case, 5, 1, 1)


def test_selection_with_non_finite_scores():
    """Infinite scores order as they are, NaN ones come last."""
    case = Case([320], 4, 2, 64, 16, "f32", seed=16, bounds=True)
    b = case.bounds
    case.q[0, :, 0] = case.q[0, :, 0].abs() + 1
    b[int(case.pages[0, 4]), :, 1, 0] = float("inf")
    b[int(case.pages[0, 9]), :, :, 0] = -float("inf")
    b[int(case.pages[0, 2]), :, :, 0] = float("nan")
    case.q[0, :, 1] = -case.q[0, :, 1].abs()
    b[int(case.pages[0, 6]), :, 1, 1] = float("inf")     # the other bound decides
    case.q[0, 0, 2] = 0
    case.q[0, 1, 2] = 0
    b[int(case.pages[0, 7]), 0, :, 2] = float("inf")     # no query reads it
    for n_select in (1, 3, 18, 19):
        check_selected(case, n_select, 0, 1 if n_select > 1 else 0)


# ----------------------------------------------------------------------------- streams, graphs

def test_repeatable_and_on_another_stream():
    import torch
    case = Case([3000, 77], 8, 2, 128, 16, "bf16", seed=17, bounds=True)
    ref = attend(case)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = case.outputs()
    ws = case.workspace()
    s.wait_stream(torch.cuda.current_stream())
    case.cache.attention(case.seqs, case.q, out, ws, lse=lse, stream=s)
    s.synchronize()
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    a, b = run_selected(case, 20, 1, 1), run_selected(case, 20, 1, 1)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_calls_follow_lengths_and_pages():
    """Two graphs over one workspace, replayed in turn with eager calls and growing sequences between them."""
    import torch
    case = Case([900, 40, 0], 8, 2, 64, 16, "bf16", seed=18, bounds=True, width=64)
    full = case.lengths.clone()
    ws = case.workspace(10)
    (o1, l1), (o2, l2) = case.outputs(), case.outputs()
    sel = torch.empty(3, 2, 10, dtype=torch.int32, device="cuda")

    def whole():
        case.cache.attention(case.seqs, case.q, o1, ws, lse=l1)

    def some():
        case.cache.attention_selected(case.seqs, case.q, o2, ws, n_select=10, lse=l2, selected=sel)

    graphs = []
    for call in (whole, some):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for step, cut in enumerate((0, 3, 39, 300)):
        case.lengths.copy_((full - cut).clamp(min=0))
        case.q.mul_(-1.0 if step else 1.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        log(f"replay with {case.lengths.tolist()}")
        check_attention(case, o1, l1)
        check_attention(case, o2, l2, chosen=choose(case, 10, 1, 1))
        eager = run_selected(case, 10, 1, 1)
        assert torch.equal(eager[0], o2) and torch.equal(eager[2], sel)


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("longest", [100, 1800])
def test_outputs_over_the_queries(heads, kv_heads, d, page, dtype, longest):
    import torch
    case = Case([longest, 1, 0, 77, longest // 2], heads, kv_heads, d, page, dtype, seed=heads + longest, bounds=True)
    ws = case.workspace(3)
    for call in (lambda q, out: case.cache.attention(case.seqs, q, out, ws),
                 lambda q, out: case.cache.attention_selected(case.seqs, q, out, ws, n_select=3)):
        out, _ = case.outputs()
        call(case.q, out)
        own = case.q.clone()
        call(own, own)
        assert torch.equal(own, out)


def test_binding_refusals():
    import torch
    case = Case([20], 4, 2, 64, 16, "bf16", seed=19)
    out, lse = case.outputs()
    ws = case.workspace()
    good = dict(seqs=case.seqs, q=case.q, out=out, workspace=ws, lse=lse)
    for kw in (dict(q=case.q.float()), dict(q=case.q[:, :3]), dict(q=case.q[:, :, :32]), dict(q=case.q.cpu()),
               dict(out=out[:0]), dict(out=out.transpose(0, 1)), dict(lse=lse.double()), dict(lse=lse[:, :2]),
               dict(workspace=ws.cpu())):
        with pytest.raises((ValueError, rk.RKError)):
            case.cache.attention(**{**good, **kw})
    with pytest.raises(rk.RKError) as e:
        case.cache.attention(**{**good, "workspace": ws[:16]})
    assert e.value.status == rk.RK_ERR_WORKSPACE
    with pytest.raises(rk.RKError):
        case.cache.attention_selected(case.seqs, case.q, out, ws, n_select=2)      # no bounds
    for bad in (case.k[:, :, ::2], case.k.transpose(2, 3), case.k.half()):
        with pytest.raises(ValueError):
            rk.PagedCache(bad, bad)
    with pytest.raises(ValueError):
        rk.PagedSeqs(case.pages.long(), case.lengths)
    with pytest.raises(ValueError):
        rk.PagedSeqs(case.pages, case.lengths[:0])
    torch.cuda.synchronize()
    assert lse.isnan().all()
