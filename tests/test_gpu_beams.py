"""The best continuations over beams and vocabulary, and the caches that follow them."""
import math

import numpy as np
import pytest

import paper_2608_08684_amd as rk
from oracle import paged as OP

from e4m3_helpers import Case8
from paged_helpers import Case, f64, torch_dtype
from test_gpu_paged_tree import make, snapshot

pytestmark = pytest.mark.gpu


def run(x, scores, n_out, ended=None, end_token=-1):
    import torch
    groups, beams = scores.shape
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    size = rk.beam_select_workspace_size(groups, beams, x.shape[1], n_out, dtype)
    assert size > 0
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    out = (torch.full((groups, n_out), -77, dtype=torch.int32, device="cuda"),
           torch.full((groups, n_out), -77, dtype=torch.int32, device="cuda"),
           torch.full((groups, n_out), 77.0, device="cuda"))
    rk.beam_select(x, scores, *out, ws, ended=ended, end_token=end_token)
    return out


def check(x, scores, n_out, out, ended=None, end_token=-1):
    """Scores: fp32 sums S of n terms in chains of n / 256 + 64 at most, exponentials good to 2^-21, one rounding at the
    end; the rest is in doubles.  Within a beam the order is that of the logits; between beams a pair may change
    places only where the exact scores are nearer than twice what log S may be off."""
    groups, beams = scores.shape
    slack = (x.shape[1] / 256 + 64) * 2.0 ** -24 + 2.0 ** -21
    logits, sc = f64(x), f64(scores)
    end = None if ended is None else ended.cpu().numpy()
    parents, tokens, best = (t.cpu().numpy() for t in out)
    for i in range(groups):
        rows = logits[i * beams:(i + 1) * beams]
        want = OP.beam_select(rows, sc[i], None if end is None else end[i], end_token, n_out)
        for j, (b, v, s) in enumerate(want):
            got = (int(parents[i, j]), int(tokens[i, j]))
            if s == -math.inf:
                assert got == (-1, -1) and best[i, j] == -np.inf, (i, j)
                continue
            assert abs(best[i, j] - s) <= slack + 2.0 ** -23 * abs(s), (i, j, best[i, j], s)
            if got != (b, v):       # only where another beam's candidate is as good
                near = [w for w in OP.beam_select(rows, sc[i], None if end is None else end[i], end_token, 4 * n_out)
                        if (w[0], w[1]) == got]
                assert near and got[0] != b and abs(near[0][2] - s) <= 2 * slack, (i, j, got, (b, v))
        assert len({(int(a), int(c)) for a, c in zip(parents[i], tokens[i]) if a >= 0}) == sum(a >= 0 for a in parents[i])


def logits(rows, vocab, dtype, seed, pad=0, shift=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g) * 3
    buf = torch.full((rows * (vocab + pad) + shift,), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    view = buf[shift:].view(rows, vocab + pad)[:, :vocab]
    view.copy_(x)
    return view


def scores_of(groups, beams, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (-5.0 * torch.rand(groups, beams, generator=g)).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups, beams, vocab, n_out", [
    (1, 1, 1, 1), (1, 1, 1, 5), (2, 3, 2, 4), (1, 4, 7, 8), (3, 2, 33, 32), (5, 4, 1000, 4), (1, 4, 50257, 4),
    (1, 1, 128256, 32), (2, 32, 32000, 32), (40, 8, 777, 16), (300, 2, 500, 2), (3, 5, 4099, 10), (1, 32, 65, 1),
    (1, 2, 600011, 8), (1, 5, 1100003, 32), (1, 1, 1 << 22, 7), (7, 16, 20000, 32),
])
def test_sizes(dtype, groups, beams, vocab, n_out):
    x, s = logits(groups * beams, vocab, dtype, vocab + n_out), scores_of(groups, beams, beams)
    check(x, s, n_out, run(x, s, n_out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_widest_call(dtype):
    """Every list of 32 beams of the longest rows."""
    import torch
    x = logits(1, 1 << 22, dtype, 1).expand(32, -1).contiguous()
    x[3, 17], x[30, -1] = 40.0, 41.0
    s = scores_of(1, 32, 2)
    out = run(x, s, 32)
    parents, tokens, best = out
    assert parents[0, 0] == 30 and tokens[0, 0] == (1 << 22) - 1 and parents[0, 1] == 3 and tokens[0, 1] == 17
    assert (best[0, 1:] <= best[0, :-1]).all() and (parents >= 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad, shift", [(0, 1), (1, 0), (3, 5), (64, 0)])
def test_rows_at_any_address(dtype, pad, shift):
    x, s = logits(12, 333, dtype, 1, pad, shift), scores_of(3, 4, 1)
    check(x, s, 6, run(x, s, 6))


@pytest.mark.parametrize("n_out", [1, 3, 8, 32])
@pytest.mark.parametrize("beams", [1, 4, 32])
def test_ties(n_out, beams):
    """Equal logits go to the lower token; rows and scores that are all the same, to the lower beam first."""
    import torch
    g = torch.Generator().manual_seed(2)
    x = torch.randint(-2, 3, (2 * beams, 900), generator=g).float()
    x[0] = 1.5
    x[beams:] = x[beams]             # the second group: one row and one score for all
    x = x.cuda()
    s = torch.zeros(2, beams, device="cuda")
    s[0] = -torch.arange(beams, device="cuda") * 0.37
    out = run(x, s, n_out)
    check(x, s, n_out, out)
    order = sorted((-float(v), b, t) for b in range(beams) for t, v in enumerate(x[beams].tolist()))[:n_out]
    # equal scores of equal rows: beam by beam; within a beam by logit, then by token
    assert [(int(a), int(t)) for a, t in zip(out[0][1], out[1][1])] == [(b, t) for _, b, t in order]


def test_ended_and_waiting_beams():
    """Ended beams have one candidate; beams with a score of -inf or NaN none, and neither's logits matter."""
    import torch
    x = logits(6 * 4, 500, "f32", 3)
    s = scores_of(6, 4, 3)
    ended = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    ended[0, 1] = ended[1, :] = ended[2, 0] = ended[5, 2] = True
    s[1] = torch.tensor([-1.0, -3.0, -1.0, -2.0])
    s[2, 1:] = -float("inf")
    s[3, 1:] = -float("inf")        # a first step
    s[4, 2] = float("nan")
    s[5] = torch.tensor([-float("inf"), float("nan"), -9.0, -float("inf")])
    s[0, 1] = 3.0                    # ended with the best score of all
    for i, b in ((0, 1), (1, 0), (3, 2), (5, 0)):
        x[i * 4 + b] = float("nan")
    for flags in (ended, ended.to(torch.uint8)):
        out = run(x, s, 6, flags, 499)
        check(x, s, 6, out, ended, 499)
    parents, tokens, best = (t.tolist() for t in out)
    assert parents[0][0] == 1 and tokens[0][0] == 499 and best[0][0] == 3.0
    assert parents[1] == [0, 2, 3, 1, -1, -1] and tokens[1] == [499] * 4 + [-1] * 2
    assert parents[2] == [0] + [-1] * 5 and parents[5] == [2] + [-1] * 5 and set(parents[3]) == {0}
    assert 2 not in parents[4]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_non_finite_logits(dtype):
    import torch
    x, s = logits(5 * 3, 700, dtype, 4), scores_of(5, 3, 4)
    x[0, 5:] = -float("inf")
    x[1] = -float("inf")
    x[2] = -float("inf")
    x[2, 699] = -3.0
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    x[6:9] = -float("inf")
    x[9, 100:] = torch.finfo(x.dtype).min
    x[10] = torch.finfo(x.dtype).min
    x[12] = 1.0e4
    out = run(x, s, 9)
    check(x, s, 9, out)
    assert (out[0][2] == -1).all()


def test_in_place_streams_and_graphs():
    import torch
    x, s = logits(4 * 4, 5000, "bf16", 5), scores_of(4, 4, 5)
    ref = run(x, s, 4)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = run(x, s, 4)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    ws = torch.empty(rk.beam_select_workspace_size(4, 4, 5000, 4, "bf16"), dtype=torch.uint8, device="cuda")
    parents, tokens, live = torch.empty_like(ref[0]), torch.empty_like(ref[1]), s.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rk.beam_select(x, live, parents, tokens, live, ws)
    live.copy_(s)
    for step in range(4):       # the scores go on from step to step
        want = run(x, live, 4)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((parents, tokens, live), want))
        x.copy_(x.roll(101, 1))


def test_beyond_32_bit_offsets():
    import torch
    vocab, rows = 128256, 9000
    buf = torch.empty(rows, vocab, device="cuda")
    x, s = logits(3, vocab, "f32", 8), scores_of(1, 3, 8)
    far = buf[rows - 1 - 2 * 4000::4000]
    far.copy_(x)
    assert all(torch.equal(a, b) for a, b in zip(run(far, s, 8), run(x, s, 8)))


def test_binding_refusals():
    import torch
    x, s = logits(6, 100, "f32", 10), scores_of(2, 3, 10)
    i, f = torch.empty(2, 4, dtype=torch.int32, device="cuda"), torch.empty(2, 4, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    e = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    for args, kw in (((x.half(), s, i, i, f, ws), {}), ((x[:5], s, i, i, f, ws), {}), ((x, s.double(), i, i, f, ws), {}),
                     ((x, s, i.long(), i, f, ws), {}), ((x, s, i, i[:, :3], f, ws), {}), ((x, s, i, i, f[:1], ws), {}),
                     ((x, s, i, i, f, ws[:64]), {}), ((x, s, i, i, f, ws.cpu()), {}),
                     ((x, s, i, i, f, ws), dict(ended=e[:, :2])), ((x, s, i, i, f, ws), dict(ended=e.int())),
                     ((x, s[0], i, i, f, ws), {}), ((x.T.contiguous().T, s, i, i, f, ws), {})):
        with pytest.raises((ValueError, rk.RKError)):
            rk.beam_select(*args, **kw)


# ----------------------------------------------------------------------------- caches of beams

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kv_heads, d, page, dtype, beams", [
    (2, 128, 16, "bf16", 4), (3, 64, 64, "bf16", 8), (2, 32, 16, "f32", 2), (1, 128, 256, "f32", 3), (2, 64, 32, "e4m3", 16),
    (8, 128, 16, "e4m3", 5), (1, 64, 16, "bf16", 32), (2, 64, 128, "f32", 17), (4, 64, 16, "bf16", 1),
])
def test_reorder(kv_heads, d, page, dtype, beams, in_place):
    """Every entry, bound and table entry after the call, for groups of any length: whole pages, one entry, none."""
    import torch
    groups = 5
    each = [3 * page + 5, 2 * page, page - 1, 1, 0]
    lengths = [n for n in each for _ in range(beams)]
    case = make([4 * page] * len(lengths), kv_heads, kv_heads, d, page, dtype, seed=beams, bounds=True)
    case.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    r = np.random.default_rng(beams)
    parents = r.integers(0, beams, (groups, beams)).astype(np.int32)
    parents[0] = np.roll(np.arange(beams), 1)           # a cycle: each page is another's source
    parents[1, ::2] = [-1, beams, -2 ** 31, 2 ** 31 - 1][beams % 4]
    held, want = snapshot(case, dtype)
    b = case.bounds.clone()
    table = case.pages.cpu().numpy()
    new, copies = OP.reordered(table, lengths, parents.ravel().tolist(), beams, page)
    # a wrong id: nothing is read there, nothing written
    if beams > 2:
        p = 2 * beams
        bad = [c for c in copies if table[p, 0] in c[:2]]
        case.pages[p, 0] = case.n_pages
        copies = [c for c in copies if c not in bad]
        new = OP.reordered(case.pages.cpu().numpy(), lengths, parents.ravel().tolist(), beams, page)[0]
    for dst, src, rest in copies:
        for t, (old, out) in enumerate(zip(held, want)):
            out[dst, :, :rest] = old[src, :, :rest]
        b[dst] = case.bounds[src]
    out = case.pages if in_place else torch.full((len(lengths), 9), -5, dtype=torch.int32, device="cuda")[:, 2:6]
    case.cache.reorder(case.seqs, torch.from_numpy(parents).cuda(), pages_out=out)
    assert out.tolist() == new
    live = torch.zeros(case.n_pages, page, dtype=torch.bool, device="cuda")     # what follows an entry in a copied
    live[:] = True                                                              # page may be anything
    for dst, _, rest in copies:
        live[dst, rest:] = False
    for got, w in zip(held, want):
        same = (got == w) | (got.isnan() & w.isnan()) if got.is_floating_point() else got == w
        at = live[:, None].expand(-1, kv_heads, -1)
        assert same[at].all()
    assert np.array_equal(f64(case.bounds), f64(b), equal_nan=True)


def test_reorder_entries_alone_and_forks():
    """Layers that share a table: entries only, then the table with the last; parents 0 fork a prompt."""
    import torch
    page, beams = 16, 3
    layers = [Case([37] * beams, 2, 2, 64, page, "bf16", seed=s) for s in (1, 1)]
    pages = layers[0].pages
    zero = torch.zeros(1, beams, dtype=torch.int32, device="cuda")
    old = [c.k.clone() for c in layers]
    before = pages.clone()
    for c, out in zip(layers, (None, pages)):
        c.cache.reorder(rk.PagedSeqs(pages, c.lengths), zero, pages_out=out)
        if out is None:
            assert torch.equal(pages, before)
    assert torch.equal(pages[:, :2], before[:1, :2].expand(beams, -1)) and torch.equal(pages[:, 2:], before[:, 2:])
    for c, k in zip(layers, old):
        for b in range(beams):
            assert torch.equal(c.k[int(pages[b, 2]), :, :5], k[int(before[0, 2]), :, :5])
    # the beams see the same cache
    c = layers[1]
    q = c.q[:1].expand(beams, -1, -1).contiguous()
    out = torch.empty_like(q)
    c.cache.attention(rk.PagedSeqs(pages, c.lengths), q, out, c.workspace())
    assert torch.equal(out[1], out[0]) and torch.equal(out[2], out[0])


def test_reorder_refusals():
    import torch
    c = Case([37] * 4, 2, 2, 64, 16, "bf16", seed=3)
    p = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    for kw in (dict(parents=p.long()), dict(parents=p[:1]), dict(parents=p.view(4)), dict(parents=p.cpu()),
               dict(parents=p.T), dict(parents=p, pages_out=c.pages.long()), dict(parents=p, pages_out=c.pages[:, :1]),
               dict(parents=p, pages_out=c.pages.T.contiguous().T)):
        with pytest.raises((ValueError, rk.RKError)):
            c.cache.reorder(c.seqs, **kw)
