"""What holds at the edges of a tree's attention, at the kernel whose waves share tiles: workgroups of 64 and 128 columns,
lengths in one part and in several.  Every test makes sure that it is that kernel."""
import pytest

import paper_2608_08684_amd as rk

import test_gpu_drafts_and_beams_chain as chain
from test_gpu_paged_tree import Drafts, make, row_type
from tree_helpers import SHARED, all_shared, lengths_of, shared

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 64), ("bf16", 128), ("e4m3", 64), ("e4m3", 128)]
forms = pytest.mark.parametrize("form", list(SHARED))
types = pytest.mark.parametrize("dtype, d", TYPES)


def run(drafts, **kw):
    with all_shared(1):
        return drafts.run(**kw)


@forms
@types
@pytest.mark.parametrize("masks", ["tree", "any", "none", None])
def test_masks(form, dtype, d, masks):
    """Trees, chains, any bits, none at all: a sequence that is its drafts alone then sees nothing."""
    case, drafts = shared(form, d, dtype, masks, seed=1)
    n, m = len(case.lens) - 1, drafts.counts[-1]
    case.lengths[n] = case.lens[n] = m
    out, lse = run(drafts)
    drafts.check(out, lse)
    if masks == "none":
        assert not out[-m:].any() and (lse[-m:] == -float("inf")).all() and lse[:-m].isfinite().all()


@types
@pytest.mark.parametrize("drafts, kv_heads", [(64, 2), (33, 3)])
def test_widest_trees_of_long_sequences(dtype, d, drafts, kv_heads):
    case = make([5000, 257, drafts, 3001], 8 * kv_heads, kv_heads, d, 32, dtype, seed=2)
    drafts = Drafts(case, [drafts, 5, drafts, 26], seed=2)
    drafts.check(*run(drafts))


@types
def test_many_sequences(dtype, d):
    n = rk.RK_MAX_BATCH_SEQS
    case = make([20 + (37 * i) % 300 for i in range(n)], 16, 2, d, 16, dtype, seed=3)
    drafts = Drafts(case, [12] + [(5 * i) % 12 for i in range(1, n)], seed=3)
    drafts.check(*run(drafts))


@forms
@types
def test_tables_with_holes_and_wrong_pages(form, dtype, d):
    case, drafts = shared(form, d, dtype, seed=6)
    last = (case.lens[0] - 1) // 16
    for i, p, bad in ((0, 0, -1), (0, 3, case.n_pages), (0, 6, 2 ** 31 - 1), (0, last, -2 ** 31), (1, 0, -7)):
        case.pages[i, p] = bad
    case.pages[-1, :] = -1
    drafts.check(*run(drafts))


@forms
@types
def test_lengths_outside(form, dtype, d):
    """Longer than the table, no longer than the drafts, zero, negative."""
    import torch
    n, most = SHARED[form][:2]
    full = {"room-64": 10240, "room-128": 4096}.get(form, 64)      # the table; the first two sequences fill it
    case, drafts = shared(form, d, dtype, seed=7, lengths=[full] * 2 + [64] * (n - 2), counts=[most] * n, table=full)
    odd = [full + 6, 2 ** 31 - 1, 3, -4, -2 ** 31, 0, 1, most][:n] if form != "room-64" else [full + 6, 3, -4]
    case.lengths[:len(odd)] = torch.tensor(odd, dtype=torch.int32)
    drafts.check(*run(drafts))


@forms
@types
@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_scale(form, dtype, d, scale):
    case, drafts = shared(form, d, dtype, seed=8)
    drafts.check(*run(drafts, scale=scale), scale=scale)


@forms
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rising", [True, False])
def test_scores_that_rise_and_fall(form, d, rising):
    """Each entry's score passes all before it by far (a column's reference moves at every tile), or none does."""
    import torch
    n = 700
    case, drafts = shared(form, d, "bf16", seed=9, lengths=[n] + lengths_of(form)[1:])
    group = case.H // 2
    q = case.q[0].view(2, group, d)[:, 0].float()
    for u in range(n):
        f = (u if rising else n - u) * 0.4 / q.norm(dim=-1, keepdim=True)
        case.k[int(case.table[0, u // 16]), :, u % 16] = (f * q).to(case.k.dtype)
    drafts.q[:drafts.counts[0], 0::2] = q.repeat_interleave(group // 2, 0).to(case.k.dtype)
    drafts.check(*run(drafts))


@forms
@types
def test_strides_and_outputs_over_the_queries(form, dtype, d):
    import torch
    case, drafts = shared(form, d, dtype, seed=10)
    ref, ref_lse = run(drafts)
    drafts.check(ref, ref_lse)
    rows, width, wide_table = len(drafts.q), case.H * d, case.pages.shape[1]
    wide = torch.full((rows, width + 64), -7.0, dtype=row_type(dtype), device="cuda")
    wide[:, 32:32 + width] = drafts.q.view(rows, -1)
    pages = torch.full((len(case.lens), wide_table + 5), 2 ** 30, dtype=torch.int32, device="cuda")
    pages[:, :wide_table] = case.pages
    seqs = rk.PagedSeqs(pages[:, :wide_table], case.lengths)
    q = wide[:, 32:32 + width].view(rows, case.H, d)
    with all_shared(1):
        case.cache.attention_tree(seqs, q, q, drafts.workspace(), drafts.offsets, masks=drafts.masks)
    assert torch.equal(q, ref) and (wide[:, :32] == -7.0).all() and (wide[:, 32 + width:] == -7.0).all()


@forms
@pytest.mark.parametrize("dtype, d, bad", [
    ("bf16", 64, float("inf")), ("bf16", 128, -float("inf")), ("bf16", 64, float("nan")), ("bf16", 128, float("nan")),
    ("e4m3", 64, float("nan")), ("e4m3", 128, float("nan")),
])
@pytest.mark.parametrize("draft", [0, 2, 9])
def test_non_finite_drafts_reach_those_who_see_them(form, dtype, d, bad, draft):
    """An infinite or NaN Value, or Key, of one draft: the rows whose mask leaves it out do not change by a bit."""
    import torch
    case, drafts = shared(form, d, dtype, seed=11)
    ref, ref_lse = run(drafts)
    channel, head, group, m = 7, 1, case.H // 2, drafts.counts[0]
    u = case.lens[0] - m + draft
    at = (int(case.table[0, u // 16]), head, u % 16, channel)
    sees = torch.zeros(len(drafts.q), dtype=torch.bool, device="cuda")
    sees[:m] = torch.tensor([bool(w >> draft & 1) for w in drafts.words[:m]])
    assert 0 < int(sees.sum()) < len(sees)
    mine = torch.zeros(case.H, dtype=torch.bool, device="cuda")
    mine[head * group:(head + 1) * group] = True
    hit = sees[:, None] & mine

    def held(name):
        return case.raw[name].view(torch.uint8) if dtype == "e4m3" else getattr(case, name)

    old = held("v")[at].clone()
    held("v")[at] = 0x7F if dtype == "e4m3" else bad
    out, lse = run(drafts)
    assert torch.equal(lse, ref_lse) and torch.equal(out[~hit], ref[~hit])
    got = out[hit][:, channel].double()
    want = torch.full_like(got, bad)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0, 1, 2), want.nan_to_num(0, 1, 2))
    rest = [x for x in range(d) if x != channel]
    assert torch.equal(out[hit][:, rest], ref[hit][:, rest])
    held("v")[at] = old
    held("k")[at] = 0x7F if dtype == "e4m3" else bad
    out, lse = run(drafts)
    assert torch.equal(out[~hit], ref[~hit]) and torch.equal(lse[~hit], ref_lse[~hit])
    assert dtype != "e4m3" or out[hit].isnan().all()


@forms
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_of_both_signs(form, d):
    case, drafts = shared(form, d, "bf16", seed=12)
    m = drafts.counts[0]
    for draft, value in ((3, float("inf")), (6, -float("inf"))):
        u = case.lens[0] - m + draft
        case.v[int(case.table[0, u // 16]), :, u % 16, 3] = value
    out, _ = run(drafts)
    kinds = set()
    for j in range(m):
        a, b = drafts.words[j] >> 3 & 1, drafts.words[j] >> 6 & 1
        got = out[j, :, 3].float()
        kinds.add((a, b))
        if a and b:
            assert got.isnan().all()
        else:
            assert (got == float("inf")).all() if a else (got == -float("inf")).all() if b else got.isfinite().all()
    assert {(0, 0), (1, 0), (0, 1)} <= kinds and out[m:].isfinite().all()


@forms
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values_of_the_text(form, d):
    """Every draft of the sequence sees them."""
    case, drafts = shared(form, d, "bf16", seed=17)
    ref, ref_lse = run(drafts)
    m, n = drafts.counts[0], case.lens[0]
    put = {0: float("inf"), d // 2 + 1: -float("inf"), d - 1: float("inf")}
    for (channel, x), u in zip(put.items(), (0, (n - m) // 2, n - m - 1)):
        case.v[int(case.table[0, u // 16]), :, u % 16, channel] = x
    out, lse = run(drafts)
    for channel, x in put.items():
        assert (out[:m, :, channel] == x).all(), channel
    rest = [x for x in range(d) if x not in put]
    assert (out[:m, :, rest] == ref[:m, :, rest]).all() and (lse == ref_lse).all() and (out[m:] == ref[m:]).all()


@types
def test_a_cache_beyond_32_bit_offsets(dtype, d):
    """5 GB of Keys; a long table makes it the shared kernel."""
    import torch
    G, page = 8, 256
    small = make([700], 32, G, d, page, dtype, seed=14, extra_pages=0, width=256)
    drafts = Drafts(small, [11], seed=14)
    ref, ref_lse = run(drafts)
    drafts.check(ref, ref_lse)
    names = ("k", "v", "k_scales", "v_scales") if dtype == "e4m3" else ("k", "v")
    held = [small.raw[n] if dtype == "e4m3" else getattr(small, n) for n in names]
    n_pages = 5 * 2 ** 30 // held[0][0].numel() // held[0].element_size()
    far, pages = [n_pages - 1, n_pages // 2, n_pages - 3], torch.full((1, 256), -1, dtype=torch.int32)
    big = []
    for t in held:
        big.append(torch.empty(n_pages, *t.shape[1:], dtype=t.dtype, device="cuda"))
        for p, to in enumerate(far):
            big[-1].view(torch.uint8)[to] = t.view(torch.uint8)[int(small.table[0, p])]
    pages[0, :3] = torch.tensor(far, dtype=torch.int32)
    cache = rk.PagedCache(*big[:2], **dict(zip(names[2:], big[2:])))
    out, lse = drafts.outputs()
    with all_shared(1):
        cache.attention_tree(rk.PagedSeqs(pages.cuda(), small.lengths), drafts.q, out, drafts.workspace(), drafts.offsets,
                             masks=drafts.masks, lse=lse)
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)


@forms
@types
def test_streams_and_graphs(form, dtype, d):
    """On another stream, and replayed from a graph while lengths and masks change."""
    import torch
    case, drafts = shared(form, d, dtype, seed=15)
    ref = run(drafts)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = run(drafts)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    out, lse = drafts.outputs()
    ws = drafts.workspace()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        case.cache.attention_tree(case.seqs, drafts.q, out, ws, drafts.offsets, masks=drafts.masks, lse=lse)
    for step in range(4):
        g.replay()
        torch.cuda.synchronize()
        eager = run(drafts)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        case.lengths.sub_(7 * step + 1)
        drafts.masks.copy_(drafts.masks.roll(1))


class Roomy(chain.Caches):
    """Tables with room for 65536 entries."""

    def __init__(self, model, n_seqs, capacity, dtype, seed=0):
        super().__init__(model, n_seqs, 1 << 16, dtype, seed)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_drafts_are_checked_kept_and_decoded_on(dtype, monkeypatch):
    """The decode loop, its prompts and its trees: of both caches' layers the prompts, and three trees."""
    monkeypatch.setattr(chain, "Caches", Roomy)
    with all_shared((2 + 3) * chain.L):
        chain.test_drafts_are_checked_kept_and_decoded_on(dtype)
