"""Drafts and beams as a decode loop uses them, over caches in bf16 and in 8 bits: a tree of drafts in one pass against the
same tokens one by one, the accepted path kept and decoded on; beams forked from one prompt, chosen and reordered step
by step against each beam's own text decoded alone.

The model is a small decoder in plain torch; every row goes through its matrices by itself, so that a token's
projections do not depend on what it is batched with."""
import math

import numpy as np
import pytest

import paper_2608_08684_amd as rk

from gpu_helpers import log

pytestmark = pytest.mark.gpu

L, H, G, D, WIDE, VOCAB, PAGE, THETA = 2, 4, 2, 64, 256, 500, 16, 1.0e4


class Model:
    def __init__(self, seed=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, scale: (torch.randn(*s, generator=g) * scale).bfloat16().float().cuda()
        self.emb = r(VOCAB, WIDE, scale=1.0)
        self.qkv = [r(WIDE, (H + 2 * G) * D, scale=WIDE ** -0.5) for _ in range(L)]
        self.o = [r(H * D, WIDE, scale=(H * D) ** -0.5) for _ in range(L)]
        self.up = [r(WIDE, 2 * WIDE, scale=WIDE ** -0.5) for _ in range(L)]
        self.down = [r(2 * WIDE, WIDE, scale=(2 * WIDE) ** -0.5) for _ in range(L)]
        self.head = r(WIDE, VOCAB, scale=3 * WIDE ** -0.5)

    @staticmethod
    def norm(h):
        import torch
        return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5)).bfloat16().float()

    @staticmethod
    def rows(x, w):
        import torch
        return torch.stack([row[None] @ w for row in x])[:, 0]


class Caches:
    """A paged cache for each layer; all layers of a sequence in pages of the same numbers, of pools of their own."""

    def __init__(self, model, n_seqs, capacity, dtype, seed=0):
        import torch
        self.m, self.n = model, n_seqs
        width = (capacity + PAGE - 1) // PAGE
        n_pages = n_seqs * width + 2
        self.caches = []
        for _ in range(L):
            if dtype == "e4m3":
                k = torch.full((n_pages, G, PAGE, D), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                s = torch.full((n_pages, G, PAGE), 255, dtype=torch.uint8, device="cuda")
                self.caches.append(rk.PagedCache(k, k.view(torch.uint8).clone().view(k.dtype), k_scales=s,
                                                 v_scales=s.clone()))
            else:
                k = torch.full((n_pages, G, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda")
                self.caches.append(rk.PagedCache(k, k.clone()))
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:n_seqs * width]
        self.pages = order.view(n_seqs, width).to(torch.int32).cuda()
        self.lengths = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
        self.seqs = rk.PagedSeqs(self.pages, self.lengths)
        c = self.caches[0]
        size = max(c.workspace_size(n_seqs, width, H), c.tree_workspace_size(n_seqs, 64 * n_seqs, width, H))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def forward(self, tokens, positions, offsets=None, masks=None):
        """Logits of new tokens: one of each sequence, or the drafts of each.  lengths counts them already."""
        import torch
        m, rows = self.m, len(tokens)
        h = m.emb[tokens.long()]
        positions = torch.as_tensor(positions, dtype=torch.int32, device="cuda")
        for l, cache in enumerate(self.caches):
            x = m.rows(m.norm(h), m.qkv[l]).bfloat16()
            q = torch.empty(rows, H, D, dtype=torch.bfloat16, device="cuda")
            out = torch.empty_like(q)
            cache.append(self.seqs, x[:, H * D:(H + G) * D].view(rows, G, D), x[:, (H + G) * D:].view(rows, G, D),
                         row_offsets=offsets, q=x[:, :H * D].view(rows, H, D), q_out=q, positions=positions,
                         rope_theta=THETA)
            if offsets is None:
                cache.attention(self.seqs, q, out, self.ws)
            else:
                cache.attention_tree(self.seqs, q, out, self.ws, offsets, masks=masks)
            h = h + m.rows(out.view(rows, -1).float(), m.o[l])
            h = h + m.rows(torch.nn.functional.silu(m.rows(m.norm(h), m.up[l])), m.down[l])
        return m.rows(m.norm(h), m.head)

    def step(self, tokens):
        import torch
        self.lengths.add_(1)
        return self.forward(torch.as_tensor(tokens).cuda(), (self.lengths - 1).tolist())


# Where two runs differ at all, an attention output was rounded to the other side of a bf16 step (or, 8-bit caches, a
# later key or value then to the other side of a step of 2^-4): at most half a step each, 2^-8 (2^-4) of a value, in a
# few values of a hundred.  As independent errors of 4 such tensors a layer, 2^-8 / sqrt(3) in one value of ten and 2^-4
# / sqrt(3) in one of a hundred, they come to sqrt(4 L) 7.2e-4 and sqrt(4 L) 3.7e-3 of the logits' 2-norm: three times that.
BOUND = {"bf16": 3 * math.sqrt(4 * L) * 7.2e-4, "e4m3": 3 * math.sqrt(4 * L) * 3.7e-3}


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_drafts_are_checked_kept_and_decoded_on(dtype):
    import torch
    model, r = Model(), np.random.default_rng(1)
    prompts, n = [[int(t) for t in r.integers(0, VOCAB, k)] for k in (37, 5, 48)], 3
    tree, alone = Caches(model, n, 160, dtype, 1), Caches(model, n, 160, dtype, 2)
    for c in (tree, alone):
        c.lengths.copy_(torch.tensor([len(p) for p in prompts], dtype=torch.int32))
        offsets = np.concatenate([[0], np.cumsum([len(p) for p in prompts])])
        # prompts of at most 64 tokens are chains of drafts
        c.forward(torch.tensor(sum(prompts, [])).cuda(), [t for p in prompts for t in range(len(p))], offsets)
    texts = [list(p) for p in prompts]
    for turn in range(3):
        counts = [12, 1, 20] if turn != 1 else [3, 17, 2]
        offsets = np.concatenate([[0], np.cumsum(counts)])
        tokens, positions, words, parents = [], [], [], []
        for i, m in enumerate(counts):
            par = [-1 if j == 0 else int(r.integers(max(-1, j - 4), j)) for j in range(m)]
            depth, word = [], []
            for j, p in enumerate(par):
                depth.append(0 if p < 0 else depth[p] + 1)
                word.append(1 << j | (0 if p < 0 else word[p]))
            parents.append(par)
            words += word
            positions += [len(texts[i]) + x for x in depth]
            tokens += [int(t) for t in r.integers(0, VOCAB, m)]
        tree.lengths.add_(torch.tensor(counts, dtype=torch.int32, device="cuda"))
        masks = torch.tensor(words, dtype=torch.int64, device="cuda")
        got = tree.forward(torch.tensor(tokens).cuda(), positions, offsets, masks)
        # the accepted path: from a root to some draft
        paths = []
        for i, par in enumerate(parents):
            j, path = int(r.integers(0, counts[i])), []
            while j >= 0:
                path.insert(0, j)
                j = par[j]
            paths.append(path)
        kept = torch.full((n, max(map(len, paths))), -1, dtype=torch.int32)
        for i, p in enumerate(paths):
            kept[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        for cache in tree.caches:
            cache.keep(tree.seqs, offsets, kept.cuda())
        tree.lengths.sub_(torch.tensor([m - len(p) for m, p in zip(counts, paths)], dtype=torch.int32, device="cuda"))
        # the same tokens one by one: each sequence's path, the others' caches left behind
        for i, path in enumerate(paths):
            for j in path:
                row = int(offsets[i]) + j
                alone.lengths[i] += 1
                one = rk.PagedSeqs(alone.pages[i:i + 1], alone.lengths[i:i + 1])
                both, alone.seqs = alone.seqs, one
                want = alone.forward(torch.tensor([tokens[row]]).cuda(), [positions[row]])[0]
                alone.seqs = both
                err = float((got[row] - want).norm() / want.norm())
                assert err < BOUND[dtype], (turn, i, j, err)
                texts[i].append(tokens[row])
        assert tree.lengths.tolist() == alone.lengths.tolist() == [len(t) for t in texts]
        # and on from there, a token each
        now = r.integers(0, VOCAB, n)
        a, b = tree.step(now), alone.step(now)
        for i in range(n):
            texts[i].append(int(now[i]))
        err = float((a - b).norm() / b.norm())
        log(f"{dtype} turn {turn}: logits {err:.2e} off in 2-norm after the path")
        assert err < BOUND[dtype]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_beams_are_forked_chosen_and_reordered(dtype):
    import torch
    model, r = Model(), np.random.default_rng(2)
    groups, beams, steps = 2, 3, 20
    n, lens = groups * beams, [30, 30]
    prompts = [[int(t) for t in r.integers(0, VOCAB, k)] for k in lens]
    c = Caches(model, n, 80, dtype, 3)
    # the prompts into each group's first sequence, then to all of its beams
    first = rk.PagedSeqs(c.pages[::beams], torch.tensor(lens, dtype=torch.int32, device="cuda"))
    every, c.seqs = c.seqs, first
    logits = c.forward(torch.tensor(sum(prompts, [])).cuda(), [t for p in prompts for t in range(len(p))],
                       np.concatenate([[0], np.cumsum(lens)]))
    c.seqs = every
    c.lengths.copy_(torch.tensor([k for k in lens for _ in range(beams)], dtype=torch.int32))
    zero = torch.zeros(groups, beams, dtype=torch.int32, device="cuda")
    for l, cache in enumerate(c.caches):
        cache.reorder(c.seqs, zero, pages_out=c.pages if l == L - 1 else None)
    logits = logits[np.cumsum(lens) - 1].repeat_interleave(beams, 0)
    scores = torch.full((groups, beams), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    parents = torch.empty(groups, beams, dtype=torch.int32, device="cuda")
    tokens = torch.empty_like(parents)
    ended = torch.zeros(groups, beams, dtype=torch.bool, device="cuda")
    ws = torch.empty(rk.beam_select_workspace_size(groups, beams, VOCAB, beams), dtype=torch.uint8, device="cuda")
    END = 7
    texts = [[[] for _ in range(beams)] for _ in range(groups)]
    for t in range(steps):
        rk.beam_select(logits, scores, parents, tokens, scores, ws, ended=ended, end_token=END)
        assert (parents >= 0).all()
        for l, cache in enumerate(c.caches):
            cache.reorder(c.seqs, parents, pages_out=c.pages if l == L - 1 else None)
        ended = ended.gather(1, parents.long()) | (tokens == END)
        texts = [[texts[i][p] + [v] for p, v in zip(ps, vs)] for i, (ps, vs) in
                 enumerate(zip(parents.tolist(), tokens.tolist()))]
        logits = c.step(tokens.view(-1).tolist())
    # every beam's text by itself
    alone = Caches(model, 1, 80, dtype, 4)
    for i in range(groups):
        for b in range(beams):
            alone.lengths.fill_(lens[i])
            out = alone.forward(torch.tensor(prompts[i]).cuda(), list(range(lens[i])), [0, lens[i]])[-1]
            total, worst = 0.0, 0.0
            for v in texts[i][b]:
                total += float(torch.log_softmax(out.double(), -1)[v])
                if v == END:
                    break
                out = alone.step([v])[0]
            # a step's log probability is off by what its logits are, of a spread of 3
            assert abs(total - float(scores[i, b])) < steps * 3 * BOUND[dtype], (i, b, total, float(scores[i, b]))
            if v != END:
                err = float((out - logits[i * beams + b]).norm() / out.norm())
                log(f"{dtype} group {i} beam {b}: score {float(scores[i, b]):.4f}, alone {total:.4f}, logits {err:.2e} off")
                assert err < BOUND[dtype]
        assert len({tuple(x) for x in texts[i]}) == beams


def test_a_captured_step_of_beams():
    """Append, attention, selection and reordering in place, replayed from a graph: as eager steps, to the last bit."""
    import torch
    groups, beams, steps = 2, 4, 20
    n = groups * beams
    g = torch.Generator().manual_seed(3)
    rows = torch.randn(steps, n, (H + 2 * G) * D, generator=g).bfloat16().cuda()

    class Side:
        def __init__(self):
            self.c = Caches(None, n, 64, "e4m3", 5)
            self.cache = self.c.caches[0]
            for t in (self.cache.k, self.cache.v):
                t.view(torch.uint8).zero_()
            self.cache.k_scales.fill_(127)
            self.cache.v_scales.fill_(127)
            self.c.lengths.fill_(9)
            self.x = torch.zeros(n, (H + 2 * G) * D, dtype=torch.bfloat16, device="cuda")
            self.q = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")
            self.out = torch.empty_like(self.q)
            self.logits = torch.zeros(n, H * D, device="cuda")
            self.scores = torch.zeros(groups, beams, device="cuda")
            self.parents = torch.zeros(groups, beams, dtype=torch.int32, device="cuda")
            self.tokens = torch.zeros_like(self.parents)
            self.ws = torch.empty(rk.beam_select_workspace_size(groups, beams, H * D, beams), dtype=torch.uint8,
                                  device="cuda")

        def step(self):
            c, x = self.c, self.x
            c.lengths.add_(1)
            self.cache.append(c.seqs, x[:, H * D:(H + G) * D].view(n, G, D), x[:, (H + G) * D:].view(n, G, D),
                              q=x[:, :H * D].view(n, H, D), q_out=self.q, rope_theta=THETA)
            self.cache.attention(c.seqs, self.q, self.out, c.ws)
            self.logits.copy_(self.out.view(n, -1))
            rk.beam_select(self.logits, self.scores, self.parents, self.tokens, self.scores, self.ws)
            self.cache.reorder(c.seqs, self.parents, pages_out=c.pages)

        def all(self):
            return (self.cache.k.view(torch.uint8), self.cache.v.view(torch.uint8), self.cache.k_scales,
                    self.cache.v_scales, self.c.pages, self.c.lengths, self.q, self.out, self.scores, self.parents,
                    self.tokens)

    eager, graphed = Side(), Side()
    start = [t.clone() for t in graphed.all()]
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        graphed.step()
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for t, s in zip(graphed.all(), start):
        t.copy_(s)
    for x in rows:
        for side in (eager, graphed):
            side.x.copy_(x)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.all(), graphed.all()))
    assert (eager.tokens >= 0).all()
