"""Appending to a paged cache against float64: rotation, places, bounds, and what must stay as it was."""
import numpy as np
import pytest

import paper_2608_08684_amd as rk
from oracle import paged as OP

from paged_helpers import f64, half_step, torch_dtype

pytestmark = pytest.mark.gpu

SHAPES = [  # heads, KV heads, head size, page, dtype
    (4, 4, 64, 16, "bf16"), (32, 8, 128, 16, "bf16"), (6, 2, 128, 64, "bf16"), (12, 12, 64, 32, "bf16"),
    (40, 40, 128, 16, "bf16"), (5, 5, 64, 256, "bf16"), (2, 2, 32, 16, "f32"), (4, 4, 64, 128, "f32"),
    (8, 2, 128, 32, "f32"), (3, 3, 32, 16, "f32"),
]


class Append:
    """lengths after the call, and how many of them are new, for each sequence."""

    def __init__(self, lengths, counts, heads, kv_heads, d, page, dtype, seed=0, bounds=True, positions=None, theta=1e4,
                 queries=True, offsets=True):
        import torch
        g = torch.Generator().manual_seed(seed)
        t = torch_dtype(dtype)
        self.__dict__.update(lens=list(lengths), counts=list(counts), H=heads, G=kv_heads, d=d, page=page, dtype=dtype,
                             theta=theta)
        n = len(lengths)
        count = [(max(x, 0) + page - 1) // page for x in lengths]
        self.n_pages = sum(count) + 4
        self.width = max(max(count), 1)
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        table = torch.full((n, self.width), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(count):
            table[i, :c] = order[at:at + c]
            at += c
        self.pages = table.cuda()
        self.lengths = torch.tensor(lengths, dtype=torch.int32).cuda()
        new = lambda *s: torch.randn(*s, generator=g).to(t).cuda()
        self.k, self.v = new(self.n_pages, kv_heads, page, d), new(self.n_pages, kv_heads, page, d)
        self.bounds = torch.stack([self.k.amin(2), self.k.amax(2)], 2) if bounds else None
        rows = sum(counts)
        self.qkv = new(rows, (heads + 2 * kv_heads) * d)
        self.q = self.qkv[:, :heads * d].view(rows, heads, d) if queries else None
        self.new_k = self.qkv[:, heads * d:(heads + kv_heads) * d].view(rows, kv_heads, d)
        self.new_v = self.qkv[:, (heads + kv_heads) * d:].view(rows, kv_heads, d)
        self.q_out = torch.full((rows, heads, d), float("nan"), dtype=t, device="cuda") if queries else None
        self.positions = None if positions is None else torch.tensor(positions(rows, g), dtype=torch.int32).cuda()
        self.offsets = [0] + np.cumsum(counts).tolist() if offsets else None

    def call(self, **kw):
        cache = rk.PagedCache(self.k, self.v, self.bounds)
        seqs = rk.PagedSeqs(self.pages, self.lengths)
        args = dict(row_offsets=self.offsets, q=self.q, q_out=self.q_out, positions=self.positions,
                    rope_theta=self.theta)
        cache.append(seqs, self.new_k, self.new_v, **{**args, **kw})

    def close(self, got, want, size):
        """One rounding of the type; fp32 angles, sines, products and their sum: 2^-21 of the pair's values."""
        err = np.abs(got - want)
        tol = half_step(self.dtype) * np.abs(want) + (2.0 ** -21 if self.theta else 0.0) * size
        assert (err <= tol).all(), (float(err.max()), np.unravel_index((err - tol).argmax(), err.shape))

    def check(self):
        """Runs the call and compares everything that it writes or must leave alone."""
        import torch
        k0, v0 = f64(self.k), f64(self.v)
        b0 = None if self.bounds is None else f64(self.bounds)
        nk, nv = f64(self.new_k), f64(self.new_v)
        qkv0 = self.qkv.clone()
        self.call()
        torch.cuda.synchronize()
        pages = self.pages.tolist()
        written, every = OP.append_rows(self.lengths.tolist(), self.counts, pages, self.page, self.n_pages)
        pos = dict(every)
        if self.positions is not None:
            pos = {r: int(self.positions[r]) for r, _ in every}
        k1, v1 = f64(self.k), f64(self.v)
        size = lambda x: np.tile(np.abs(x[..., :self.d // 2]) + np.abs(x[..., self.d // 2:]), 2)
        untouched = np.ones(k0.shape[:1] + (self.page,), bool)
        for r, p, s in written:
            untouched[p, s] = False
            self.close(k1[p, :, s], OP.rotate(nk[r], pos[r], self.theta), size(nk[r]))
            assert np.array_equal(v1[p, :, s], nv[r])
        assert np.array_equal(k1.transpose(0, 2, 1, 3)[untouched], k0.transpose(0, 2, 1, 3)[untouched])
        assert np.array_equal(v1.transpose(0, 2, 1, 3)[untouched], v0.transpose(0, 2, 1, 3)[untouched])
        if b0 is not None:
            want, slots = b0.copy(), {}
            for _, p, s in written:
                slots.setdefault(p, []).append(s)
            for p, s in slots.items():      # of the keys as they were stored
                lo, hi = k1[p, :, s].min(0), k1[p, :, s].max(0)
                if 0 not in s:
                    lo, hi = np.minimum(lo, b0[p, :, 0]), np.maximum(hi, b0[p, :, 1])
                want[p, :, 0], want[p, :, 1] = lo, hi
            assert np.array_equal(f64(self.bounds), want)
        if self.q is not None:
            q = f64(self.q)
            for r, _ in every:
                self.close(f64(self.q_out[r]), OP.rotate(q[r], pos[r], self.theta), size(q[r]))
        assert torch.equal(self.qkv, qkv0)


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
def test_one_row_each(heads, kv_heads, d, page, dtype):
    lens = [1, 2, page, page + 1, 2 * page - 1, 5, 0, 3 * page]
    Append(lens, [1] * 8, heads, kv_heads, d, page, dtype, offsets=False).check()


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
def test_prompts_and_chunks(heads, kv_heads, d, page, dtype):
    """Whole prompts, chunks that start and end inside pages, no rows, more rows than entries (the first ones have no
    place)."""
    lens = [3 * page + 7, 40, 1, 2 * page + 3, page, 9, 70]
    counts = [3 * page + 7, 17, 1, 5, page, 0, 33]
    Append(lens, counts, heads, kv_heads, d, page, dtype, seed=1).check()
    Append([5, 0, 3], [9, 2, 3], heads, kv_heads, d, page, dtype, seed=2).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(dtype):
    """Angles of positions up to 2^31 - 1 and of negative ones."""
    pos = lambda n, g: [0, 1, -1, 131071, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31][:n]
    Append([8] * 4, [2] * 4, 4, 2, 64, 16, dtype, seed=3, positions=pos, theta=5.0e5).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rotation_copies(dtype):
    Append([40, 7], [40, 3], 4, 2, 64, 16, dtype, seed=4, theta=0.0).check()


def test_without_queries_or_bounds():
    Append([40, 7], [40, 3], 4, 2, 128, 16, "bf16", seed=5, queries=False).check()
    Append([40, 7], [40, 3], 4, 2, 128, 16, "bf16", seed=6, bounds=False).check()
    Append([40, 7], [1, 1], 4, 2, 128, 16, "bf16", seed=7, queries=False, bounds=False, offsets=False).check()


def test_rows_without_a_place():
    """Pages outside the cache and entries past the table take nothing; the queries are rotated all the same."""
    import torch
    a = Append([50, 33, 64, 20], [50, 33, 40, 20], 4, 2, 64, 16, "bf16", seed=8)
    a.pages[0, 1] = -1
    a.pages[1, 2] = a.n_pages
    a.pages[3, :] = 2 ** 31 - 1
    a.lengths[2] = 64 + 11      # of a table of 4 pages
    a.check()
    b = Append([50, 33, 20], [1, 1, 1], 4, 2, 64, 16, "f32", seed=9, offsets=False)
    b.lengths.copy_(torch.tensor([-3, 2 ** 31 - 1, 20], dtype=torch.int32))
    b.positions = torch.tensor([4, 5, 6], dtype=torch.int32).cuda()
    b.check()


def test_queries_in_place():
    import torch
    a = Append([40, 7], [40, 3], 8, 2, 128, 16, "bf16", seed=10)
    a.call()
    b = Append([40, 7], [40, 3], 8, 2, 128, 16, "bf16", seed=10)
    b.call(q_out=b.q)
    assert torch.equal(b.q, a.q_out) and torch.equal(b.k, a.k) and torch.equal(b.new_k, a.new_k)


def test_head_major_rows():
    """Blocks [KV head][row][head_dim], as the selection with budgets leaves them."""
    import torch
    a = Append([40], [40], 4, 2, 64, 16, "bf16", seed=11, theta=0.0, queries=False)
    blocks_k = a.new_k.transpose(0, 1).contiguous()
    blocks_v = a.new_v.transpose(0, 1).contiguous()
    b = Append([40], [40], 4, 2, 64, 16, "bf16", seed=11, theta=0.0, queries=False)
    b.new_k, b.new_v = blocks_k.transpose(0, 1), blocks_v.transpose(0, 1)
    a.call()
    b.call()
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.bounds, b.bounds)


@pytest.mark.parametrize("dtype, page", [("bf16", 16), ("bf16", 64), ("f32", 32)])
def test_growing_by_pieces_is_growing_at_once(dtype, page):
    """The same rows in one call, in chunks and one by one leave the same cache and bounds, to the last bit."""
    import torch
    total = 2 * page + 9
    ref = Append([total], [total], 4, 2, 64, page, dtype, seed=12)
    ref.call()
    for step in (1, 7, page, page + 3):
        a = Append([total], [total], 4, 2, 64, page, dtype, seed=12)
        cache, seqs = rk.PagedCache(a.k, a.v, a.bounds), rk.PagedSeqs(a.pages, a.lengths)
        for r in range(0, total, step):
            m = min(step, total - r)
            a.lengths.fill_(r + m)
            cache.append(seqs, a.new_k[r:r + m], a.new_v[r:r + m], row_offsets=None if m == 1 else [0, m],
                         q=a.q[r:r + m], q_out=a.q_out[r:r + m], rope_theta=1e4)
        for x, y in ((a.k, ref.k), (a.v, ref.v), (a.bounds, ref.bounds), (a.q_out, ref.q_out)):
            assert torch.equal(x, y), step


def test_captured_steps_follow_lengths():
    """One captured step replayed token by token, with eager work between, against eager steps."""
    import torch
    a, b = (Append([30, 5], [1, 1], 4, 2, 64, 16, "bf16", seed=13, offsets=False) for _ in range(2))
    ca, sa = rk.PagedCache(a.k, a.v, a.bounds), rk.PagedSeqs(a.pages, a.lengths)
    for x in (a, b):
        x.pages.copy_(torch.tensor([[0, 1], [2, 3]], dtype=torch.int32))
        x.lengths.copy_(torch.tensor([14, 1], dtype=torch.int32))
    # the capture's warm-up writes what its first replay writes again
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ca.append(sa, a.new_k, a.new_v, q=a.q, q_out=a.q_out, rope_theta=1e4)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ca.append(sa, a.new_k, a.new_v, q=a.q, q_out=a.q_out, rope_theta=1e4)
    for _ in range(6):
        g.replay()
        b.call()
        torch.cuda.synchronize()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.bounds, b.bounds), (a.q_out, b.q_out)):
            assert torch.equal(x, y)
        for x in (a, b):
            x.lengths.add_(1)
            x.qkv.mul_(-1.5)


def test_binding_refusals():
    import torch
    a = Append([40, 7], [40, 3], 4, 2, 64, 16, "bf16", seed=14)
    k0 = a.k.clone()
    for kw in (dict(q=None), dict(q_out=None), dict(row_offsets=[0, 43]), dict(row_offsets=[0, 40, 42]),
               dict(row_offsets=None), dict(positions=torch.zeros(43, dtype=torch.int64, device="cuda")),
               dict(positions=torch.zeros(42, dtype=torch.int32, device="cuda")), dict(q=a.q.float()),
               dict(q=a.q[:, :3]), dict(rope_theta=0.5)):
        with pytest.raises((ValueError, rk.RKError)):
            a.call(**kw)
    cache, seqs = rk.PagedCache(a.k, a.v, a.bounds), rk.PagedSeqs(a.pages, a.lengths)
    for k, v in ((a.new_k.cpu(), a.new_v), (a.new_k[:, :1], a.new_v), (a.new_k, a.new_v.float()),
                 (a.new_k[:, :, ::2], a.new_v)):
        with pytest.raises(ValueError):
            cache.append(seqs, k, v, row_offsets=a.offsets)
    torch.cuda.synchronize()
    assert torch.equal(a.k, k0)
