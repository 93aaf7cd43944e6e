"""Attention of drafted tokens over a paged cache against float64, and the path that is kept of them."""
import math

import numpy as np
import pytest

import paper_2608_08684_amd as rk
from oracle import paged as OP

from e4m3_helpers import Case8
from paged_helpers import Case, attention_tolerance, f64, torch_dtype

pytestmark = pytest.mark.gpu


def make(lengths, heads, kv_heads, d, page, dtype, seed=0, **kw):
    if dtype == "e4m3":
        return Case8(lengths, heads, kv_heads, d, page, seed=seed, **kw)
    return Case(lengths, heads, kv_heads, d, page, dtype, seed=seed, **kw)


def row_type(dtype):
    return torch_dtype("f32" if dtype == "f32" else "bf16")


class Drafts:
    """Queries and masks of the last counts[i] entries of each sequence of a case."""

    def __init__(self, case, counts, masks="tree", seed=0):
        import torch
        self.case, self.counts = case, list(counts)
        self.offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        rows = int(self.offsets[-1])
        g = torch.Generator().manual_seed(seed + 100)
        self.q = torch.randn(rows, case.H, case.d, generator=g).mul_(2.0).to(case.q.dtype).cuda()
        r = np.random.default_rng(seed)
        self.words = []
        for m in counts:
            own = []
            for j in range(m):
                if masks == "tree":
                    p = int(r.integers(max(-1, j - 5), j)) if j else -1
                    own.append(1 << j | (own[p] if p >= 0 else 0))
                elif masks == "any":         # any bits, those of no draft too
                    own.append(int(r.integers(0, 1 << 63)) * 2 + int(r.integers(0, 2)))
                elif masks == "none":
                    own.append(0)
                else:
                    own.append((2 << j) - 1)
            self.words += own
        self.masks = None if masks is None else torch.tensor(np.array(self.words, np.uint64).view(np.int64)).cuda()

    def outputs(self):
        import torch
        rows = len(self.q)
        return (torch.full_like(self.q, float("nan")), torch.full((rows, self.case.H), float("nan"), device="cuda"))

    def workspace(self):
        import torch
        n, c = len(self.counts), self.case
        size = c.cache.tree_workspace_size(n, len(self.q), c.seqs.max_pages, c.H)
        assert size > 0
        return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, **kw):
        out, lse = self.outputs()
        self.case.cache.attention_tree(self.case.seqs, self.q, out, self.workspace(), self.offsets, masks=self.masks,
                                       lse=lse, **kw)
        return out, lse

    def check(self, out, lse, scale=0.0):
        """The tolerance of the one-token attention holds: its weights' two bf16 parts, and a score's own rounding of
        (d + 8) 2^-24 of the summed |q k|, which is more than the 3 roundings of its exponent (factor, product and
        difference, 2^-24 of numbers no larger than 1.5 times the score and 64 each: under 2^-16 together for weights
        above e^-40).  A log-sum-exp adds a product of its reference, at most 1.5 |lse| + 64 in units of log 2, with a
        rounded log 2 and a sum: 2^-23 of that."""
        c = self.case
        scale = scale or 1.0 / math.sqrt(c.d)
        grp, entries = c.H // c.G, c.seqs.max_pages * c.page
        out, lse, q = f64(out), f64(lse), f64(self.q)
        k_all, v_all = f64(c.k), f64(c.v)
        pages = c.pages.cpu().numpy()
        for i, m in enumerate(self.counts):
            for j in range(m):
                r = int(self.offsets[i]) + j
                at = [(int(pages[i, u // c.page]), u % c.page)
                      for u in OP.visible(int(c.lengths[i]), m, self.words[r], entries)]
                at = [x for x in at if 0 <= x[0] < c.n_pages]
                p, s = [x[0] for x in at], [x[1] for x in at]
                for g in range(c.G):
                    h = slice(g * grp, (g + 1) * grp)
                    o, l, weighted, products = OP.attend(q[r, h], k_all[p, g, s], v_all[p, g, s], scale)
                    tol, ltol = attention_tolerance(c.dtype, len(at), c.d, scale, o, weighted, products)
                    err = np.abs(out[r, h] - o)
                    assert (err <= tol).all(), (i, j, g, len(at), float(err.max()), float(tol.flat[err.argmax()]))
                    if not at:
                        assert (lse[r, h] == -np.inf).all() and not out[r, h].any()
                    else:
                        assert (np.abs(lse[r, h] - l) <= ltol + 2.0 ** -23 * (64 + 3.5 * np.abs(l))).all(), (i, j, g)


SHAPES = [  # heads, KV heads, head size, page, dtype
    (4, 4, 64, 16, "bf16"), (8, 2, 128, 16, "bf16"), (6, 2, 128, 64, "e4m3"), (35, 1, 64, 16, "bf16"),
    (4, 4, 64, 256, "e4m3"), (16, 2, 128, 32, "e4m3"), (2, 2, 32, 16, "f32"), (4, 4, 64, 16, "f32"),
    (8, 2, 128, 32, "f32"), (12, 12, 64, 128, "bf16"),
]
SHORT = [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 130, 64, 9]


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("masks", ["tree", "any", None])
def test_short_lengths(heads, kv_heads, d, page, dtype, masks):
    """From a sequence that is its drafts alone to more than a tile's text before them; a sequence without any."""
    case = make(SHORT, heads, kv_heads, d, page, dtype, seed=heads)
    drafts = Drafts(case, [1, 1, 15, 3, 17, 5, 16, 33, 64, 1, 20, 13, 0], masks, seed=1)
    drafts.check(*drafts.run())


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("counts", [[5, 1, 7, 3], [40, 64, 3, 26]])
def test_long_lengths_are_split_and_joined(heads, kv_heads, d, page, dtype, counts):
    case = make([5000, 64, 257, 3001], heads, kv_heads, d, page, dtype, seed=2)
    drafts = Drafts(case, counts, seed=2)
    drafts.check(*drafts.run())


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("lengths, counts", [
    ([9000, 300, 4100, 1], [8, 5, 3, 1]),    # 32 columns a KV head over long caches: waves with one block of them
    ([3000], [64]),                          # 256 columns, parts of 128 entries
    ([1500], [61]),                          # 244 columns, 16 a workgroup
    ([4090, 3000], [26, 11]),                # fewer parts than 512 workgroups would be
])
def test_lengths_and_widths_between(dtype, lengths, counts):
    case = make(lengths, 32, 8, 128, 64 if dtype == "e4m3" else 16, dtype, seed=len(lengths))
    drafts = Drafts(case, counts, seed=4)
    drafts.check(*drafts.run())


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_many_sequences(dtype):
    n = rk.RK_MAX_BATCH_SEQS
    case = make([20 + (37 * i) % 300 for i in range(n)], 4, 2, 64, 16, dtype, seed=3)
    drafts = Drafts(case, [(5 * i) % 12 for i in range(n)], seed=3)
    drafts.check(*drafts.run())


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_rows_that_see_nothing(dtype):
    """Drafts alone, and masks without a bit: zeros, a log-sum-exp of -inf."""
    case = make([5, 40, 64], 4, 2, 64, 16, dtype, seed=4)
    drafts = Drafts(case, [5, 40, 3], "none", seed=4)
    out, lse = drafts.run()
    drafts.check(out, lse)
    assert not out[:45].any() and (lse[:45] == -float("inf")).all() and lse[45:].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_tables_with_holes_and_lengths_outside(dtype):
    import torch
    case = make([100, 500, 64, 900, 64], 4, 2, 64, 16, dtype, seed=6, width=60)
    for i, p, bad in ((0, 0, -1), (0, 6, case.n_pages), (1, 3, 2 ** 31 - 1), (1, 31, -2 ** 31), (3, 56, -7)):
        case.pages[i, p] = bad
    case.pages[2, :] = -1
    drafts = Drafts(case, [9, 20, 5, 17, 10], seed=6)
    drafts.check(*drafts.run())
    # longer than the table, no longer than the drafts, negative
    case = make([64, 64, 64, 64, 64], 4, 2, 64, 16, dtype, seed=7, width=4)
    case.lengths.copy_(torch.tensor([70, 2 ** 31 - 1, 3, -4, -2 ** 31], dtype=torch.int32))
    drafts = Drafts(case, [10, 5, 10, 5, 64], seed=7)
    drafts.check(*drafts.run())


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 32), ("e4m3", 64)])
@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_scale(dtype, d, scale):
    case = make([300, 40], 8, 2, d, 16, dtype, seed=8)
    drafts = Drafts(case, [9, 30], seed=8)
    drafts.check(*drafts.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rising", [True, False])
def test_scores_that_rise_and_fall(dtype, rising):
    """Each entry's score passes all before it by far (a column's reference moves at every tile), or none does."""
    import torch
    n = 700
    case = make([n], 4, 2, 64, 16, dtype, seed=9)
    q = case.q[0].view(2, 2, 64)[:, 0].float()
    for u in range(n):
        f = (u if rising else n - u) * 0.4 / q.norm(dim=-1, keepdim=True)
        case.k[int(case.table[0, u // 16]), :, u % 16] = (f * q).to(case.k.dtype)
    drafts = Drafts(case, [20], seed=9)
    drafts.q[:, 0::2] = q.to(case.k.dtype)
    out, lse = drafts.run()
    drafts.check(out, lse)


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("f32", 64), ("e4m3", 64)])
def test_strides_and_outputs_over_the_queries(dtype, d):
    import torch
    case = make([77, 300, 31], 8, 2, d, 16, dtype, seed=10)
    drafts = Drafts(case, [20, 3, 31], seed=10)
    ref, ref_lse = drafts.run()
    drafts.check(ref, ref_lse)
    rows, t = len(drafts.q), row_type(dtype)
    wide = torch.full((rows, 8 * d + 64), -7.0, dtype=t, device="cuda")
    wide[:, 32:32 + 8 * d] = drafts.q.view(rows, -1)
    pages = torch.full((3, case.pages.shape[1] + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    pages[:, :case.pages.shape[1]] = case.pages
    seqs = rk.PagedSeqs(pages[:, :case.pages.shape[1]], case.lengths)
    q = wide[:, 32:32 + 8 * d].view(rows, 8, d)
    case.cache.attention_tree(seqs, q, q, drafts.workspace(), drafts.offsets, masks=drafts.masks)
    assert torch.equal(q, ref) and (wide[:, :32] == -7.0).all() and (wide[:, 32 + 8 * d:] == -7.0).all()


@pytest.mark.parametrize("dtype, bad", [("bf16", float("inf")), ("bf16", -float("inf")), ("bf16", float("nan")),
                                        ("f32", float("inf")), ("f32", -float("inf")), ("f32", float("nan")),
                                        ("e4m3", float("nan"))])
@pytest.mark.parametrize("heads", [4, 16])
def test_non_finite_drafts_reach_those_who_see_them(dtype, bad, heads):
    """An infinite or NaN Value, or Key, of one draft: the rows whose mask leaves it out do not change by a bit."""
    import torch
    case = make([70, 90], heads, 2, 64, 16, dtype, seed=11)
    drafts = Drafts(case, [10, 30], seed=11)
    ref, ref_lse = drafts.run()
    draft, channel, head = 4, 7, 1
    u = 90 - 30 + draft
    page, slot = int(case.table[1, u // 16]), u % 16
    sees = torch.tensor([i == 1 and bool(drafts.words[int(drafts.offsets[i]) + j] >> draft & 1)
                         for i in range(2) for j in range(drafts.counts[i])]).cuda()
    assert 0 < int(sees.sum()) < 30
    grp = heads // 2
    mine = torch.zeros(heads, dtype=torch.bool, device="cuda")
    mine[head * grp:(head + 1) * grp] = True
    hit = sees[:, None] & mine

    def put(name):
        if dtype == "e4m3":
            case.raw[name].view(torch.uint8)[page, head, slot, channel] = 0x7F
        else:
            getattr(case, name)[page, head, slot, channel] = bad

    old = (case.raw["v"].view(torch.uint8) if dtype == "e4m3" else case.v)[page, head, slot, channel].clone()
    put("v")
    out, lse = drafts.run()
    assert torch.equal(lse, ref_lse)
    assert torch.equal(out[~hit], ref[~hit])
    got = out[hit][:, channel].double()
    want = torch.full_like(got, bad)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0, 1, 2), want.nan_to_num(0, 1, 2))
    rest = [x for x in range(64) if x != channel]
    assert torch.equal(out[hit][:, rest], ref[hit][:, rest])
    (case.raw["v"].view(torch.uint8) if dtype == "e4m3" else case.v)[page, head, slot, channel] = old
    put("k")
    out, lse = drafts.run()
    assert torch.equal(out[~hit], ref[~hit]) and torch.equal(lse[~hit], ref_lse[~hit])


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", [
    (4, 4, 64, 16, "bf16"), (8, 2, 128, 16, "bf16"), (24, 1, 64, 32, "bf16"), (4, 2, 32, 16, "f32"), (8, 2, 128, 64, "f32"),
])
@pytest.mark.parametrize("lengths, counts", [([700, 40], [3, 1]), ([5000, 1300], [40, 24])])
def test_infinite_values_of_the_text(heads, kv_heads, d, page, dtype, lengths, counts):
    """Every draft sees them, and a weight is positive however small: their channels are those infinities."""
    case = make(lengths, heads, kv_heads, d, page, dtype, seed=17)
    drafts = Drafts(case, counts, seed=17)
    ref, ref_lse = drafts.run()
    put = {0: float("inf"), d // 2 + 1: -float("inf"), d - 1: float("inf")}
    for i, n in enumerate(lengths):
        for (channel, x), u in zip(put.items(), (0, (n - counts[i]) // 2, n - counts[i] - 1)):
            case.v[int(case.table[i, u // page]), :, u % page, channel] = x
    out, lse = drafts.run()
    for channel, x in put.items():
        assert (out[:, :, channel] == x).all(), channel
    rest = [x for x in range(d) if x not in put]
    assert (out[:, :, rest] == ref[:, :, rest]).all() and (lse == ref_lse).all()


@pytest.mark.parametrize("drafts, heads", [(2, 4), (12, 8), (40, 16)])   # 4, 48 and 320 columns a KV head
@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_infinite_values_of_small_weight(drafts, heads, dtype, d):
    """A weight of e^-50 of the largest."""
    case = make([2048] * 4, heads, 2, d, 16, dtype, seed=18)
    case.k.zero_()
    for i in range(4):
        case.k[int(case.table[i, 0]), :, 0, 0] = 5.0
        for channel, u, x in ((3, 1, float("inf")), (d - 2, 1700, -float("inf"))):
            case.v[int(case.table[i, u // 16]), :, u % 16, channel] = x
    rows = Drafts(case, [drafts] * 4, seed=18)
    rows.q.zero_()
    rows.q[:, :, 0] = 10.0
    out, lse = rows.run(scale=1.0)
    assert (out[:, :, 3] == float("inf")).all() and (out[:, :, d - 2] == -float("inf")).all()
    assert (lse == 50.0).all()
    rest = [x for x in range(d) if x not in (3, d - 2)]
    assert out[:, :, rest].isfinite().all()


def test_infinities_of_both_signs():
    import torch
    case = make([90], 4, 2, 64, 16, "bf16", seed=12)
    drafts = Drafts(case, [30], seed=12)
    for draft, value in ((4, float("inf")), (7, -float("inf"))):
        u = 60 + draft
        case.v[int(case.table[0, u // 16]), :, u % 16, 3] = value
    out, _ = drafts.run()
    for j in range(30):
        a, b = drafts.words[j] >> 4 & 1, drafts.words[j] >> 7 & 1
        got = out[j, :, 3].float()
        if a and b:
            assert got.isnan().all()
        else:
            assert (got == float("inf")).all() if a else (got == -float("inf")).all() if b else got.isfinite().all()


def test_one_draft_is_the_attention_of_one_token():
    """A sequence with a single draft: what rk_paged_attention gives, to the tolerance of either."""
    case = Case([300, 5000, 17], 8, 2, 128, 16, "bf16", seed=13)
    drafts = Drafts(case, [1, 1, 1], None, seed=13)
    drafts.q = case.q
    out, lse = drafts.run()
    drafts.check(out, lse)


def test_a_cache_beyond_32_bit_offsets():
    import torch
    G, d, page = 8, 128, 256
    n_pages = 5 * 2 ** 30 // (G * page * d * 2)
    k = torch.empty(n_pages, G, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Case([700], 16, G, d, page, "bf16", seed=14, extra_pages=0)
    drafts = Drafts(small, [11], seed=14)
    ref, ref_lse = drafts.run()
    drafts.check(ref, ref_lse)
    at = [n_pages - 1, n_pages // 2, n_pages - 3]
    for p, far in enumerate(at):
        k[far], v[far] = small.k[int(small.table[0, p])], small.v[int(small.table[0, p])]
    seqs = rk.PagedSeqs(torch.tensor([at], dtype=torch.int32, device="cuda"), small.lengths)
    out, lse = drafts.outputs()
    rk.PagedCache(k, v).attention_tree(seqs, drafts.q, out, drafts.workspace(), drafts.offsets, masks=drafts.masks,
                                       lse=lse)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)


def test_streams_and_graphs():
    """On another stream, and replayed from a graph while lengths and masks change."""
    import torch
    case = make([3000, 200, 64], 8, 2, 128, 16, "bf16", seed=15)
    drafts = Drafts(case, [12, 30, 5], seed=15)
    ref = drafts.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = drafts.run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    out, lse = drafts.outputs()
    ws = drafts.workspace()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        case.cache.attention_tree(case.seqs, drafts.q, out, ws, drafts.offsets, masks=drafts.masks, lse=lse)
    for step in range(3):
        g.replay()
        torch.cuda.synchronize()
        eager = drafts.run()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        case.lengths.sub_(7 * step + 1)
        drafts.masks.copy_(drafts.masks.roll(1))


def test_binding_refusals():
    import torch
    case = make([64, 64], 4, 2, 64, 16, "bf16", seed=16)
    drafts = Drafts(case, [3, 4], seed=16)
    out, lse = drafts.outputs()
    ws = drafts.workspace()
    good = dict(q=drafts.q, out=out, workspace=ws, row_offsets=drafts.offsets, masks=drafts.masks, lse=lse)
    case.cache.attention_tree(case.seqs, **good)
    for bad in (dict(q=drafts.q.float()), dict(q=drafts.q[:6]), dict(out=out[:, :2]), dict(row_offsets=[0, 7]),
                dict(row_offsets=[0, 3, 8]), dict(row_offsets=[0, 8, 7]), dict(masks=drafts.masks.int()),
                dict(masks=drafts.masks[:5]), dict(masks=drafts.masks.cpu()), dict(lse=lse.double()),
                dict(q=drafts.q.transpose(0, 1).contiguous().transpose(0, 1)), dict(workspace=ws.cpu())):
        with pytest.raises((ValueError, rk.RKError)):
            case.cache.attention_tree(case.seqs, **{**good, **bad})
    kept = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for args in ((drafts.offsets, kept.long()), (drafts.offsets, kept[:1]), (drafts.offsets, kept.cpu()),
                 (drafts.offsets, kept.T.contiguous().T), ([0, 7], kept), (drafts.offsets, kept[:, :0]),
                 ([0, 3, 70], kept)):
        with pytest.raises((ValueError, rk.RKError)):
            case.cache.keep(case.seqs, *args)


# ----------------------------------------------------------------------------- the path that is kept

def snapshot(case, dtype):
    import torch
    held = [case.raw[n] for n in ("k", "v", "k_scales", "v_scales")] if dtype == "e4m3" else [case.k, case.v]
    held = [t.view(torch.uint8) if t.element_size() == 1 else t for t in held]
    return held, [t.clone() for t in held]


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("bounds", [True, False])
def test_keep(heads, kv_heads, d, page, dtype, bounds):
    """Every entry of the caches after the call: the path's moved, all else to the bit as it was."""
    import torch
    lengths = [64, 65, 70, 100, 33, 20, 17, 300, 90, 64]
    counts = [64, 64, 30, 26, 1, 20, 5, 40, 7, 0]
    case = make(lengths, heads, kv_heads, d, page, dtype, seed=20, bounds=bounds)
    kept = torch.full((10, 64), -1, dtype=torch.int32)
    paths = [list(range(64)), list(range(1, 64, 2)), [0, 1, 2, 20, 29], [25], [0], [3, 9, 19], [], [5, 4, 6],
             [0, 3, 7, 8], [0]]
    for i, p in enumerate(paths):
        kept[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
    if page == 16:
        case.pages[8, 5] = -1       # all of its drafts on no page
        case.pages[3, 4] = -1       # the path's new entry alone
    held, want = snapshot(case, dtype)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    b = None if case.bounds is None else f64(case.bounds)
    keys = f64(case.k)
    table = case.pages.cpu().numpy()
    for i, (n, m) in enumerate(zip(lengths, counts)):
        fresh = {}
        for dst, src in OP.kept_moves(n, m, paths[i]):
            (p, s), (q, t) = [(int(table[i, e // page]), e % page) for e in (dst, src)]
            if p < 0 or q < 0:
                continue
            for new, old in zip(want, held):
                new[p, :, s] = old[q, :, t]
            fresh.setdefault(p, []).append((s, keys[q, :, t]))
        for p, rows in fresh.items():
            if b is not None:
                x = np.stack([r for _, r in rows])
                anew = any(s == 0 for s, _ in rows)
                b[p, :, 0] = x.min(0) if anew else np.minimum(x.min(0), b[p, :, 0])
                b[p, :, 1] = x.max(0) if anew else np.maximum(x.max(0), b[p, :, 1])
    case.cache.keep(case.seqs, offsets, kept.cuda())
    for got, new in zip(held, want):
        same = (got == new) | (got.isnan() & new.isnan()) if got.is_floating_point() else got == new
        assert same.all()
    if b is not None:
        assert np.array_equal(f64(case.bounds), b, equal_nan=True)


def test_keep_rows_that_are_strided_and_short():
    """kept as columns of a wider row; a path longer than n_kept is cut to it."""
    import torch
    case = make([40, 50], 4, 2, 64, 16, "bf16", seed=21)
    ref = case.k.clone()
    wide = torch.full((2, 9), 7, dtype=torch.int32, device="cuda")
    wide[:, 1:4] = torch.tensor([[1, 3, 5], [2, 3, 9]], dtype=torch.int32)
    case.cache.keep(case.seqs, [0, 10, 20], wide[:, 1:3])
    row = lambda t, i, e: t[int(case.table[i, e // 16]), :, e % 16]
    for i, b, path in ((0, 30, (1, 3)), (1, 40, (2, 3))):
        for j, t in enumerate(path):
            assert torch.equal(row(case.k, i, b + j), row(ref, i, b + t))
        assert all(torch.equal(row(case.k, i, b + j), row(ref, i, b + j)) for j in range(2, 10))
