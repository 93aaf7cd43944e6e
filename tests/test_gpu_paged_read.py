"""Rows read back out of the paged cache, in all forms of the call and of the cache: copies, compared bit by bit."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk

from paged_helpers import Case, torch_dtype
from test_gpu_paged_tree import make

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 64), ("bf16", 128), ("f32", 32), ("f32", 64), ("f32", 128), ("e4m3", 64), ("e4m3", 128)]
types = pytest.mark.parametrize("dtype, d", TYPES)
LENGTHS = [1, 15, 16, 17, 64, 130, 33, 0, 300]


def row_type(dtype):
    return torch_dtype("f32" if dtype == "f32" else "bf16")


def expected(case, counts, name):
    """The rows [sum of counts, KV heads, d]: entry by entry from the tables; 0 where there is no page."""
    import torch
    held, table, lengths = getattr(case, name), case.pages.cpu().numpy(), case.lengths.tolist()
    out = torch.zeros(sum(counts), case.G, case.d, dtype=held.dtype, device="cuda")
    r = 0
    for i, m in enumerate(counts):
        for j in range(m):
            e = lengths[i] - m + j
            if 0 <= e < table.shape[1] * case.page and 0 <= table[i, e // case.page] < case.n_pages:
                out[r] = held[int(table[i, e // case.page]), :, e % case.page]
            r += 1
    return out


def buffer(case, rows, layout):
    """(whole buffer, a view [rows, KV heads, d] of it): filled with -7."""
    import torch
    G, d, t = case.G, case.d, case.k.dtype
    if layout == "rows":
        whole = torch.full((rows, G, d), -7.0, dtype=t, device="cuda")
        return whole, whole
    if layout == "heads first":
        whole = torch.full((G, rows + 1, d), -7.0, dtype=t, device="cuda")
        return whole, whole[:, 1:].transpose(0, 1)
    whole = torch.full((rows, 3 * G * d + 16), -7.0, dtype=t, device="cuda")      # columns of a fused row
    return whole, whole[:, 8:8 + G * d + 8 * G].view(rows, G, d + 8)[:, :, :d]


def same(a, b):
    """Equal bits, but for a NaN's (a row of 8 bits has one NaN of each sign)."""
    import torch
    assert a.shape == b.shape
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check(case, counts, layout="rows", names="kv", offsets=True):
    rows = sum(counts)
    bufs = {n: buffer(case, rows, layout) for n in names}
    case.cache.read(case.seqs, **{n: v for n, (_, v) in bufs.items()},
                    row_offsets=np.concatenate([[0], np.cumsum(counts)]) if offsets else None)
    for n, (whole, view) in bufs.items():
        assert same(view, expected(case, counts, n)), n
        view.fill_(-7.0)                # nothing beside the rows was written
        assert (whole == -7.0).all(), n
    return bufs


@types
@pytest.mark.parametrize("kv_heads, page", [(1, 16), (3, 64), (8, 256)])
@pytest.mark.parametrize("layout", ["rows", "heads first", "fused"])
def test_one_row_each(dtype, d, kv_heads, page, layout):
    """The last entry of each sequence; an empty one has none."""
    case = make(LENGTHS, kv_heads, kv_heads, d, page, dtype, seed=1)
    check(case, [1] * len(LENGTHS), layout, offsets=False)


@types
@pytest.mark.parametrize("kv_heads, page", [(1, 256), (3, 16), (8, 32)])
@pytest.mark.parametrize("layout", ["rows", "heads first", "fused"])
def test_ranges(dtype, d, kv_heads, page, layout):
    """Whole sequences, their ends, none of them, and more rows than there are entries."""
    case = make(LENGTHS, kv_heads, kv_heads, d, page, dtype, seed=2)
    check(case, [1, 15, 5, 0, 64, 100, 40, 3, 290], layout)


@types
@pytest.mark.parametrize("names", ["k", "v"])
@pytest.mark.parametrize("offsets", [True, False])
def test_keys_or_values_alone(dtype, d, names, offsets):
    case = make(LENGTHS, 2, 2, d, 16, dtype, seed=3)
    check(case, [1, 9, 16, 2, 64, 1, 33, 0, 299] if offsets else [1] * len(LENGTHS), names=names, offsets=offsets)


@types
@pytest.mark.parametrize("offsets", [True, False])
def test_holes_and_lengths_outside(dtype, d, offsets):
    """Pages that are none, lengths beyond the table and negative ones: those entries are 0."""
    import torch
    lengths = [100, 500, 64, 300, 64, 64, 64, 64]
    case = make(lengths, 2, 2, d, 16, dtype, seed=4)
    for i, p, bad in ((0, 0, -1), (0, 6, case.n_pages), (1, 3, 2 ** 31 - 1), (1, 31, -2 ** 31), (3, 18, -7)):
        case.pages[i, p] = bad
    case.pages[2, :] = -1
    case.lengths[4:] = torch.tensor([16 * case.pages.shape[1] + 3, 2 ** 31 - 1, -4, -2 ** 31], dtype=torch.int32)
    check(case, [100, 130, 64, 40, 20, 5, 7, 9] if offsets else [1] * 8, offsets=offsets)


@types
def test_many_rows(dtype, d):
    """More than 16 workgroups to a CU's worth of rows: several of them a workgroup."""
    lengths = [9000, 1, 4097]
    case = make(lengths, 2, 2, d, 64, dtype, seed=5)
    check(case, lengths)


def test_no_rows():
    import torch
    case = Case([5, 0], 2, 2, 64, 16, "bf16", seed=6)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    case.cache.read(case.seqs, none, none, row_offsets=[0, 0, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_beyond_32_bit_offsets(dtype):
    """Pages whose offsets in bytes and in elements need more than 32 bits."""
    import torch
    G, d, page = 8, 128, 256
    n_pages = (2 ** 32 + 2 ** 28) // (G * page * d)
    k = torch.empty(n_pages, G, page, d, dtype=row_type(dtype), device="cuda")
    rows = torch.randn(700, G, d, generator=torch.Generator().manual_seed(7)).to(k.dtype).cuda()
    at = [n_pages - 1, n_pages // 2, n_pages - 3]
    for p, far in enumerate(at):
        part = rows[p * page:(p + 1) * page]
        k[far, :, :len(part)] = part.transpose(0, 1)
    seqs = rk.PagedSeqs(torch.tensor([at], dtype=torch.int32, device="cuda"),
                        torch.tensor([700], dtype=torch.int32, device="cuda"))
    out = torch.empty_like(rows)
    rk.PagedCache(k, k).read(seqs, out, row_offsets=[0, 700])
    assert torch.equal(out, rows)
    one = torch.empty_like(rows[:1])
    rk.PagedCache(k, k).read(seqs, None, one)
    assert torch.equal(one, rows[-1:])


@types
def test_streams_and_graphs(dtype, d):
    """On another stream, and replayed from a graph while the lengths change."""
    import torch
    case = make([300, 70, 33], 2, 2, d, 16, dtype, seed=8)
    counts, offsets = [20, 5, 33], [0, 20, 25, 58]
    k, v = (buffer(case, 58, "rows")[0] for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        case.cache.read(case.seqs, k, v, row_offsets=offsets)
    s.synchronize()
    assert same(k, expected(case, counts, "k")) and same(v, expected(case, counts, "v"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        case.cache.read(case.seqs, k, v, row_offsets=offsets)
    for step in range(4):
        k.fill_(-7.0)
        v.fill_(-7.0)
        g.replay()
        torch.cuda.synchronize()
        assert same(k, expected(case, counts, "k")) and same(v, expected(case, counts, "v"))
        case.lengths.sub_(9 * step + 1)


@types
def test_binding_refusals(dtype, d):
    import torch
    case = make([20, 30], 2, 2, d, 16, dtype, seed=9)
    good = torch.empty(2, 2, d, dtype=row_type(dtype), device="cuda")
    other = torch.float32 if dtype != "f32" else torch.bfloat16
    for kw in (dict(), dict(k=good.to(other)), dict(v=good[:1]), dict(k=good.cpu()), dict(k=good[:, :, :d // 2]),
               dict(v=good.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=good, row_offsets=[0, 1]),
               dict(k=good, row_offsets=[0, 2, 1]), dict(k=good, row_offsets=[1, 1, 2]),
               dict(k=torch.empty(2, 2, d + 1, dtype=good.dtype, device="cuda")[:, :, :d]),
               dict(k=good.flatten()[:d].expand(2, 2, d))):
        with pytest.raises((ValueError, rk.RKError)):
            case.cache.read(case.seqs, **kw)
