"""Paged caches of 8-bit values: quantised as they are written, read back, attended to."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk
from oracle import paged as OP

from e4m3_helpers import Case8, empty_cache, rounded, values
from paged_helpers import Case, check_attention, f64

pytestmark = pytest.mark.gpu


def seqs_of(table, lengths):
    import torch
    return rk.PagedSeqs(torch.tensor(table, dtype=torch.int32, device="cuda"),
                        torch.tensor(lengths, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("d", [64, 128])
def test_every_code_under_every_scale(d):
    """All 256 codes with scales 2^-117 .. 2^120 read back as the numbers that they stand for."""
    import torch
    page, per = 256, 256 // d
    cache = empty_cache(per, 1, page, d)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(per, 1, 1, d).expand(-1, 1, page, -1)
    cache.k.view(torch.uint8).copy_(codes)
    cache.v.view(torch.uint8).copy_(codes.flip(-1))
    scales = torch.arange(page, device="cuda").clamp(10, 247).to(torch.uint8)
    cache.k_scales.copy_(scales.expand(per, 1, -1))
    cache.v_scales.copy_(scales.flip(0).expand(per, 1, -1))
    seqs = seqs_of([list(range(per))], [per * page])
    k = torch.empty(per * page, 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache.read(seqs, k, v, row_offsets=[0, per * page])
    for got, held, sc in ((k, cache.k, cache.k_scales), (v, cache.v, cache.v_scales)):
        want = values(held, sc)[:, 0].reshape(-1, d)
        want = torch.where(want.abs() >= 2.0 ** 128, want.sign() * float("inf"), want)   # beyond bf16
        same = (f64(got[:, 0]) == want.cpu().numpy()) | (np.isnan(f64(got[:, 0])) & want.isnan().cpu().numpy())
        assert same.all()


def hard_rows(d):
    """Rows at which the rounding and the scale can go wrong, as bf16 [rows, d]."""
    import torch
    g = torch.Generator().manual_seed(1)
    rows = [torch.randn(d, generator=g) * 2.0 ** e for e in (-130, -126, -118, -117, -40, -9, -1, 0, 1, 7, 8, 9, 60, 118)]
    rows += [torch.zeros(d), torch.full((d,), 2.0 ** -133), torch.full((d,), 3.38e38)]
    for top in (1.75, 1.7578125, 1.7421875, 1.0, 1.9921875):          # next to where the scale changes
        for e in (-119, -3, 0, 5, 127):
            r = torch.randn(d, generator=g).clamp(-1, 1) * 2.0 ** (e - 3)
            r[d // 3] = -top * 2.0 ** e
            rows.append(r)
    ties = torch.tensor([(2 * i + 1) * 2.0 ** (j - 5) for i in range(8, 16) for j in range(8)])   # half way, all steps
    rows.append(torch.cat([ties, -ties])[:d].clone())
    rows[-1][0] = 448.0
    small = torch.arange(d) * 2.0 ** -10                                # below the least normal number, halves too
    small[5] = 300.0
    rows.append(small)
    for bad in (float("inf"), -float("inf"), float("nan")):
        r = torch.randn(d, generator=g)
        r[7] = bad
        rows.append(r)
    rows.append(torch.full((d,), float("nan")))
    return torch.stack(rows).bfloat16().cuda()


@pytest.mark.parametrize("d", [64, 128])
def test_rounding_of_rows(d):
    """Without a rotation: the codes and scales of the definition, to the bit; what reads back are their values."""
    import torch
    x = hard_rows(d)
    n, G, page = len(x), 3, 16
    cache = empty_cache((n + page - 1) // page + 1, G, page, d, bounds=True)
    width = (n + page - 1) // page
    seqs = seqs_of([list(range(width))], [n])
    k = torch.stack([x, x.flip(0), x.roll(3, 0)], 1)
    v = k.flip(1).contiguous()
    cache.append(seqs, k, v, row_offsets=[0, n])
    back_k, back_v = torch.empty_like(k), torch.empty_like(v)
    cache.read(seqs, back_k, back_v, row_offsets=[0, n])
    for rows, held, scales, back in ((k, cache.k, cache.k_scales, back_k), (v, cache.v, cache.v_scales, back_v)):
        codes, sc = rounded(rows)
        got = held.view(torch.uint8).transpose(1, 2).reshape(-1, G, d)[:n]
        nan = codes.float().isnan()
        want = codes.view(torch.uint8)
        assert ((got == want) | (nan & (got & 0x7F == 0x7F))).all()
        assert torch.equal(scales.transpose(1, 2).reshape(-1, G)[:n], sc)
        exact = values(codes, sc)
        assert torch.equal(back.double().isnan(), nan) and torch.equal(back.double()[~nan], exact[~nan])
        for r in range(0, n, 5):        # the definition, value by value
            units, byte = OP.e4m3(f64(rows[r, 0]))
            assert byte == int(sc[r, 0]) and np.array_equal(np.float64(units), f64(codes[r, 0].float()), equal_nan=True)
    # what no row went to
    assert (cache.k_scales[-1] == 0).all() and (cache.k.view(torch.uint8)[-1] == 0x7F).all()
    # bounds: of the values that the page holds, NaN where one is
    exact = values(*rounded(k))
    for p in range(width):
        part = exact[p * page:(p + 1) * page]
        lo, hi = part.amin(0), part.amax(0)             # torch keeps a NaN
        b = cache.key_bounds[p].double()
        assert torch.equal(b[:, 0].isnan(), lo.isnan()) and torch.equal(b[:, 0].nan_to_num(7.0), lo.nan_to_num(7.0))
        assert torch.equal(b[:, 1].isnan(), hi.isnan()) and torch.equal(b[:, 1].nan_to_num(7.0), hi.nan_to_num(7.0))


def check_rotated(cache, seqs, k, counts, positions, theta):
    """Rotated keys: within half a step of the exact rotation, which fp32 has to 2^-21 of the pair's size; the scale that
    of the largest value to 2^-20."""
    import torch
    page, n_pages = cache.page_size, len(cache.k)
    held, scales = f64(values(cache.k, cache.k_scales)), cache.k_scales.cpu().numpy()
    x = f64(k)
    written, _ = OP.append_rows(seqs.lengths.tolist(), counts, seqs.pages.tolist(), page, n_pages)
    for row, p, slot in written:
        y = OP.rotate(x[row], int(positions[row]), theta)
        half = x.shape[-1] // 2
        size = np.hypot(x[row][:, :half], x[row][:, half:])
        slack = np.concatenate([size, size], -1) * 2.0 ** -21
        for h in range(x.shape[1]):
            top, unit = np.abs(y[h]).max(), 2.0 ** (int(scales[p, h, slot]) - 127)
            assert 224 * unit * (1 - 2.0 ** -20) < top <= 448 * unit * (1 + 2.0 ** -20)
            assert (np.abs(held[p, h, slot] - y[h]) <= np.maximum(np.abs(y[h]) / 16, unit * 2.0 ** -10) + slack[h]).all()
    return written


@pytest.mark.parametrize("G, d, page, lengths, counts", [
    (8, 128, 16, [1, 17, 300, 64, 5], None), (1, 64, 64, [7, 64, 65], None),
    (2, 128, 32, [100, 33, 0, 31], [100, 20, 0, 31]), (12, 64, 16, [40, 3], [25, 3]), (3, 64, 256, [700], [700]),
])
def test_append_rotates_and_rounds(G, d, page, lengths, counts):
    import torch
    g = torch.Generator().manual_seed(2)
    width = (max(lengths) + page - 1) // page
    n_pages = width * len(lengths) + 2
    cache = empty_cache(n_pages, G, page, d, bounds=True)
    table = torch.randperm(n_pages, generator=g)[:width * len(lengths)].view(len(lengths), width)
    seqs = seqs_of(table.tolist(), lengths)
    offsets = None if counts is None else np.concatenate([[0], np.cumsum(counts)])
    rows, H = len(lengths) if counts is None else int(offsets[-1]), 2 * G
    k, v = (torch.randn(rows, G, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(rows, H, d, generator=g).bfloat16().cuda()
    q_out, q_ref = torch.empty_like(q), torch.empty_like(q)
    positions = torch.randint(0, 100000, (rows,), generator=g).to(torch.int32).cuda()
    cache.append(seqs, k, v, row_offsets=offsets, q=q, q_out=q_out, positions=positions, rope_theta=1e4)
    written = check_rotated(cache, seqs, k, [1] * len(lengths) if counts is None else counts, positions.tolist(), 1e4)
    codes, sc = rounded(v)
    for row, p, slot in written:
        assert torch.equal(cache.v.view(torch.uint8)[p, :, slot], codes.view(torch.uint8)[row])
        assert torch.equal(cache.v_scales[p, :, slot], sc[row])
    at = torch.zeros(n_pages, page, dtype=torch.bool)
    for _, p, slot in written:
        at[p, slot] = True
    rest = ~at.cuda()[:, None].expand(-1, G, -1)
    assert (cache.k_scales[rest] == 0).all() and (cache.v.view(torch.uint8)[rest] == 0x7F).all()
    # the queries: what a bf16 cache's append makes of them
    big = torch.empty(n_pages, G, page, d, dtype=torch.bfloat16, device="cuda")
    rk.PagedCache(big, torch.empty_like(big)).append(seqs, k, v, row_offsets=offsets, q=q, q_out=q_ref,
                                                     positions=positions, rope_theta=1e4)
    assert torch.equal(q_out, q_ref)
    # bounds, of pages begun anew
    got, held = f64(cache.key_bounds), f64(values(cache.k, cache.k_scales))
    for p in sorted({p for _, p, slot in written if slot == 0}):
        slots = [s for _, pp, s in written if pp == p]
        assert np.array_equal(got[p, :, 0], held[p][:, slots].min(1)) and np.array_equal(got[p, :, 1], held[p][:, slots].max(1))


def test_steps_extend_the_bounds():
    """Row by row: a page's bounds are those of its rows so far."""
    import torch
    g = torch.Generator().manual_seed(3)
    G, d, page = 2, 64, 16
    cache = empty_cache(4, G, page, d, bounds=True)
    seqs = seqs_of([[2, 0], [3, 1]], [0, 5])
    seqs.lengths.zero_()
    for t in range(20):
        seqs.lengths.add_(1)
        k = torch.randn(2, G, d, generator=g).bfloat16().cuda()
        cache.append(seqs, k, k, rope_theta=1e4)
        held, b = f64(values(cache.k, cache.k_scales)), f64(cache.key_bounds)
        for p in ((2, 3) if t < 16 else (0, 1)):
            rows = held[p][:, :t % page + 1]
            assert np.array_equal(b[p, :, 0], rows.min(1)) and np.array_equal(b[p, :, 1], rows.max(1))


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200]
SHAPES = [(8, 2, 128, 16), (6, 2, 128, 64), (16, 1, 64, 256), (20, 1, 128, 32), (35, 1, 64, 16), (12, 12, 64, 32)]


@pytest.mark.parametrize("heads, kv_heads, d, page", SHAPES)
@pytest.mark.parametrize("lengths", [EDGES, [5000, 0, 1, 257, 4096, 3001], [(7 * i) % 91 for i in range(300)]],
                         ids=["edges", "long", "many"])
def test_attention(heads, kv_heads, d, page, lengths):
    """Against float64 over the values that the cache stands for.  (A bf16 cache of them gives the same but for the order
    in which a score's d products are added: 8-bit rows come 16 channels to a lane, bf16 ones 8.  Either order is
    within the tolerance's (d + 8) 2^-24 of the summed |q k|.)"""
    case = Case8(lengths, heads, kv_heads, d, page, seed=heads)
    out, lse = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace(), lse=lse)
    check_attention(case, out, lse)


@pytest.mark.parametrize("lengths, select", [([700, 33, 0, 1000], 7), ([20000, 300], 9), ([9], 3), ([40000] * 2, 1100)])
def test_selected_pages(lengths, select):
    """The pages that a bf16 cache with the same bounds chooses, and float64 over them."""
    import torch
    case = Case8(lengths, 8, 2, 64, 16, seed=5, bounds=True)
    got = []
    for cache in (case.cache, case.plain):
        out, lse = case.outputs()
        chosen = torch.empty(len(lengths), 2, select, dtype=torch.int32, device="cuda")
        cache.attention_selected(case.seqs, case.q, out, case.workspace(select), n_select=select, keep_last=2, lse=lse,
                                 selected=chosen)
        got.append((out, lse, chosen))
    assert torch.equal(got[0][2], got[1][2])
    chosen = [[[p for p in row if p >= 0] for row in rows] for rows in got[0][2].tolist()]
    check_attention(case, *got[0][:2], chosen=chosen)


def test_non_finite_rows_stay_with_their_sequence():
    import torch
    case = Case8([50, 50, 50], 4, 2, 64, 16, seed=9)
    ref, _ = case.outputs()
    case.cache.attention(case.seqs, case.q, ref, case.workspace())
    case.raw["v"].view(torch.uint8)[int(case.table[1, 1]), 0, 3, 7] = 0xFF
    case.raw["k"].view(torch.uint8)[int(case.table[2, 0]), 1, 2, 5] = 0x7F
    out, _ = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace())
    assert (out[0] == ref[0]).all() and (out[1, 2:] == ref[1, 2:]).all() and (out[2, :2] == ref[2, :2]).all()
    assert out[1, :2, 7].isnan().all() and out[2, 2:].isnan().all()
    keep = [x for x in range(64) if x != 7]
    assert (out[1, :2][:, keep] == ref[1, :2][:, keep]).all()


def test_tables_with_holes_and_wrong_pages():
    case = Case8([100, 500, 64, 900, 33], 4, 2, 64, 16, seed=6)
    for i, p, bad in ((0, 0, -1), (0, 6, case.n_pages), (1, 3, 2 ** 31 - 1), (1, 4, -2 ** 31), (3, 56, -7)):
        case.pages[i, p] = bad
    case.pages[2, :] = -1
    out, lse = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace(), lse=lse)
    check_attention(case, out, lse)


def test_a_cache_beyond_32_bit_offsets():
    """Pages whose byte offsets need more than 32 bits, written, read back and attended to."""
    import torch
    G, d, page = 8, 128, 256
    n_pages = 5 * 2 ** 30 // (G * page * d)
    big = empty_cache(n_pages, G, page, d)
    small = empty_cache(3, G, page, d)
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(700, G, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(1, 16, d, generator=g).bfloat16().cuda()
    got = []
    for cache, pages in ((big, [n_pages - 1, n_pages // 2, n_pages - 3]), (small, [2, 0, 1])):
        seqs = seqs_of([pages], [700])
        cache.append(seqs, k, v, row_offsets=[0, 700], rope_theta=1e4)
        kb, vb, out = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
        cache.read(seqs, kb, vb, row_offsets=[0, 700])
        ws = torch.empty(cache.workspace_size(1, 3, 16), dtype=torch.uint8, device="cuda")
        cache.attention(seqs, q, out, ws)
        got.append((kb, vb, out))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and (got[0][0] != 0).any()


def test_binding_refusals():
    import torch
    cache = empty_cache(2, 2, 16, 64)
    s = cache.k_scales
    for args, kw in (((cache.k, cache.v), {}), ((cache.k, cache.v), dict(k_scales=s)),
                     ((cache.k, cache.k.float().bfloat16()), dict(k_scales=s, v_scales=s)),
                     ((cache.k, cache.v), dict(k_scales=s.int(), v_scales=s)),
                     ((cache.k, cache.v), dict(k_scales=s[:1], v_scales=s)),
                     ((cache.k, cache.v, torch.empty(2, 2, 2, 64, device="cuda")), dict(k_scales=s, v_scales=s)),
                     ((cache.k.float().bfloat16(),) * 2, dict(k_scales=s, v_scales=s)),
                     ((cache.k.view(torch.uint8),) * 2, dict(k_scales=s, v_scales=s))):
        with pytest.raises(ValueError):
            rk.PagedCache(*args, **kw)
    seqs = seqs_of([[0, 1]], [3])
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(k=x.float(), v=x.float()), dict(k=x.to(torch.float8_e4m3fn), v=x)):
        with pytest.raises(ValueError):
            cache.append(seqs, **kw)
    for kw in (dict(), dict(k=x.float()), dict(k=x[:, :1]), dict(v=x.cpu()), dict(k=x, row_offsets=[0, 2]),
               dict(k=x, row_offsets=[0, 1, 1])):
        with pytest.raises((ValueError, rk.RKError)):
            cache.read(seqs, **kw)
