"""The serving operators as a decode loop uses them: prompt caches cut to per-layer budgets, moved to pages, grown token
by token, attended to, and the logits scored.

The same tokens over the same compressed caches are what rk_policy_damage evaluates as a window, so its logits are the
reference; the rest of the decoder (norms, projections, feed-forward) is plain torch in float32 on the same bf16
weights.
"""
import numpy as np
import pytest

import fixtures as F
import paper_2608_08684_amd as rk

from gpu_helpers import Runner, empty_bytes, log, make_batch

pytestmark = pytest.mark.gpu


class Decoder:
    """One-token steps of the library's decoder; each layer's cache in pages of its own pool."""

    def __init__(self, cfg, weights, n_seqs, capacity, page, bounds=True):
        import torch
        self.cfg, self.n = cfg, n_seqs
        bf = lambda t: t.view(torch.bfloat16).float()
        self.w = {k: [bf(x) for x in weights[k]] for k in ("w_qkv", "w_o", "w_gate_up", "w_down")}
        self.emb, self.head = bf(weights["tok_emb"]), bf(weights["lm_head"])
        self.norms = weights
        width = (capacity + page - 1) // page
        n_pages = n_seqs * width + 1
        g = torch.Generator().manual_seed(1)
        new = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.caches, self.seqs = [], []
        for _ in range(cfg.n_layers):
            k = new(n_pages, cfg.n_kv_heads, page, cfg.head_dim)
            b = new(n_pages, cfg.n_kv_heads, 2, cfg.head_dim) if bounds else None
            self.caches.append(rk.PagedCache(k, torch.full_like(k, float("nan")), b))
            pages = torch.randperm(n_pages, generator=g)[:n_seqs * width].view(n_seqs, width).to(torch.int32).cuda()
            self.seqs.append(rk.PagedSeqs(pages, torch.zeros(n_seqs, dtype=torch.int32, device="cuda")))
        H = cfg.n_heads
        size = max(c.workspace_size(n_seqs, width, H, width) for c in self.caches)
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.q = torch.empty(n_seqs, H, cfg.head_dim, dtype=torch.bfloat16, device="cuda")
        self.out = torch.empty_like(self.q)

    def fill(self, layer, i, k, v):
        """Retained Keys and Values [KV head][entry][head_dim] of sequence i: rotated already."""
        s = self.seqs[layer]
        s.lengths[i] = k.shape[1]
        one = rk.PagedSeqs(s.pages[i:i + 1], s.lengths[i:i + 1])
        self.caches[layer].append(one, k.transpose(0, 1), v.transpose(0, 1), row_offsets=[0, k.shape[1]])

    def norm(self, h, gain):
        import torch
        return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + self.cfg.rms_eps) * gain).bfloat16().float()

    def step(self, tokens, position, attend=None):
        """Logits [n, vocab] of one token per sequence at the given text position."""
        import torch
        c = self.cfg
        H, G, d = c.n_heads, c.n_kv_heads, c.head_dim
        h = self.emb[tokens.long()]
        positions = torch.full((self.n,), position, dtype=torch.int32, device="cuda")
        for l in range(c.n_layers):
            qkv = (self.norm(h, self.norms["attn_norm"][l]) @ self.w["w_qkv"][l].T).bfloat16()
            self.seqs[l].lengths.add_(1)
            self.caches[l].append(self.seqs[l], qkv[:, H * d:(H + G) * d].view(self.n, G, d),
                                  qkv[:, (H + G) * d:].view(self.n, G, d), q=qkv[:, :H * d].view(self.n, H, d),
                                  q_out=self.q, positions=positions, rope_theta=c.rope_theta)
            (attend or self.whole)(l)
            h = h + self.out.view(self.n, -1).float() @ self.w["w_o"][l].T
            gate, up = (self.norm(h, self.norms["mlp_norm"][l]) @ self.w["w_gate_up"][l].T).chunk(2, -1)
            h = h + (torch.nn.functional.silu(gate) * up).bfloat16().float() @ self.w["w_down"][l].T
        return self.norm(h, self.norms["final_norm"]) @ self.head.T

    def whole(self, l):
        self.caches[l].attention(self.seqs[l], self.q, self.out, self.ws)

    def all_pages(self, l):
        self.caches[l].attention_selected(self.seqs[l], self.q, self.out, self.ws, n_select=self.seqs[l].max_pages)


@pytest.mark.parametrize("heads, kv_heads, head_dim, P, budgets, page", [
    (8, 2, 128, 300, [90, 45, 300], 16),      # grouped queries; the last layer keeps its prompt whole
    (4, 4, 64, 517, [33, 200], 32),
])
def test_decoding_over_compressed_caches(heads, kv_heads, head_dim, P, budgets, page):
    """Window logits against rk_policy_damage's.  Roundings to bf16 on the way, each 2^-9 / sqrt(3) of its tensor's
    size: 6 per layer and the final norm there, 7 (the rows before their rotation) and one here; as independent they
    come to sqrt(13 L + 2) 1.13e-3 of the logits' 2-norm, and the bound is three times that.  The bounds' pages,
    all of them chosen, give the same to the joining's rounding."""
    import torch
    n, W, w = 2, 5, 16
    L = len(budgets)
    cfg = F.small_model(n_layers=L, d_model=256, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, d_ff=512,
                        vocab=1024, dtype="bf16")
    run = Runner(cfg, F.make_weights(cfg))
    m = run.model
    toks = F.make_tokens(F.make_workload("chain", cfg, [P + W] * n, seed_id=77))
    # the compressed prompt caches
    prompts = make_batch([t[:P] for t in toks])
    state = empty_bytes(m.snapkv_state_size(prompts.rows, n, w))
    ws = empty_bytes(m.snapkv_workspace_size(prompts.rows, n, w))
    m.snapkv_prefill(prompts, w, state, ws)
    total, offs = rk.snapkv_layout(prompts, L, [budgets] * n)
    pos = torch.empty(kv_heads * total, dtype=torch.int32, device="cuda")
    k = torch.empty(kv_heads * total, head_dim, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    m.snapkv_compress(prompts, [budgets] * n, state, pos, k, v, ws, obs_window=w)
    # the reference: the window's tokens over the retained positions
    batch = make_batch(toks)
    wstate = empty_bytes(m.window_state_size(batch.rows))
    ws = empty_bytes(m.workspace_size(batch.rows, 1, rk.RK_FLAG_CACHED_WINDOW | rk.RK_FLAG_UNFUSED_KL))
    m.window_reference(batch, P, wstate, ws)
    d = torch.empty(n, device="cuda")
    want = torch.empty(n * W, cfg.vocab, device="cuda")
    before = np.concatenate([[0], np.cumsum(budgets)])
    m.policy_damage(batch, P, pos, [int(kv_heads * b) for b in before[:-1]], int(kv_heads * before[-1]), budgets,
                    wstate, d, ws, logits_out=want)
    want = want.view(n, W, -1)
    for attend in ("whole", "all_pages"):
        dec = Decoder(cfg, run.dw, n, max(budgets) + W, page)
        for i in range(n):
            for l in range(L):
                keep = budgets[l]
                e0 = int(offs[i * L + l]) * kv_heads
                block = slice(e0, e0 + kv_heads * keep)
                dec.fill(l, i, k[block].view(kv_heads, keep, head_dim), v[block].view(kv_heads, keep, head_dim))
        lp, ent = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        rank = torch.empty(n, dtype=torch.int32, device="cuda")
        ids, tops = torch.empty(n, 5, dtype=torch.int32, device="cuda"), torch.empty(n, 5, device="cuda")
        lws = empty_bytes(rk.token_logprobs_workspace_size(n, cfg.vocab, 5))
        for t in range(W):
            now = torch.tensor([int(x[P + t]) for x in toks], dtype=torch.int32, device="cuda")
            got = dec.step(now, P + t, getattr(dec, attend))
            err = float((got - want[:, t]).norm() / want[:, t].norm())
            log(f"{attend} step {t}: logits {err:.2e} off in 2-norm")
            assert err < 3 * 1.13e-3 * (13 * L + 2) ** 0.5
            # the next tokens' log probabilities, from both sides' logits
            nxt = torch.tensor([int(x[min(P + t + 1, P + W - 1)]) for x in toks], dtype=torch.int32, device="cuda")
            for logits in (got, want[:, t].contiguous()):
                rk.token_logprobs(logits, nxt, lws, logprob=lp, rank=rank, entropy=ent, top_ids=ids, top_logprobs=tops)
                exact = torch.log_softmax(logits.double(), -1)
                assert (lp - exact.gather(1, nxt.long()[:, None])[:, 0]).abs().max() < 2e-5
                assert (ent + (exact.exp() * exact).sum(-1)).abs().max() < 2e-5
                assert torch.equal(ids.long(), exact.argsort(dim=-1, descending=True, stable=True)[:, :5])
                assert (tops - exact.gather(1, ids.long())).abs().max() < 2e-5
        for l in range(L):
            assert dec.seqs[l].lengths.tolist() == [budgets[l] + W] * n


class Side:
    """The buffers of a decode step and the step: append, attention over selected pages, log probabilities."""

    def __init__(self, n, H, G, d, page):
        import torch
        self.n, self.H, self.G, self.d = n, H, G, d
        self.qkv = torch.empty(n, (H + 2 * G) * d, dtype=torch.bfloat16, device="cuda")
        k = torch.zeros(3 * n + 1, G, page, d, dtype=torch.bfloat16, device="cuda")
        self.cache = rk.PagedCache(k, k.clone(), torch.zeros(3 * n + 1, G, 2, d, dtype=k.dtype, device="cuda"))
        self.seqs = rk.PagedSeqs(torch.arange(3 * n, dtype=torch.int32, device="cuda").view(n, 3),
                                 torch.tensor([0, 7, 30], dtype=torch.int32, device="cuda") % 28)
        self.q = torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda")
        self.out, self.lse = torch.empty_like(self.q), torch.empty(n, H, device="cuda")
        self.ws = torch.empty(self.cache.workspace_size(n, 3, H, 2), dtype=torch.uint8, device="cuda")
        self.logits = torch.empty(n, H * d, device="cuda")
        self.tok = torch.tensor([1, 2, 511], dtype=torch.int32, device="cuda")
        self.lp, self.ent = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        self.ids = torch.empty(n, 9, dtype=torch.int32, device="cuda")
        self.lws = torch.empty(rk.token_logprobs_workspace_size(n, H * d, 9), dtype=torch.uint8, device="cuda")

    def step(self):
        x, n, H, G, d = self.qkv, self.n, self.H, self.G, self.d
        self.seqs.lengths.add_(1)
        self.cache.append(self.seqs, x[:, H * d:(H + G) * d].view(n, G, d), x[:, (H + G) * d:].view(n, G, d),
                          q=x[:, :H * d].view(n, H, d), q_out=self.q, rope_theta=1e4)
        self.cache.attention_selected(self.seqs, self.q, self.out, self.ws, n_select=2, lse=self.lse)
        self.logits.copy_(self.out.view(n, -1))      # any numbers that follow from the step
        rk.token_logprobs(self.logits, self.tok, self.lws, logprob=self.lp, entropy=self.ent, top_ids=self.ids)

    def all(self):
        return (self.cache.k, self.cache.v, self.cache.key_bounds, self.q, self.out, self.lse, self.lp, self.ent,
                self.ids, self.seqs.lengths)


def test_the_steps_of_a_loop_as_one_graph():
    """A captured decode step (append, attention, log probabilities) replayed: the same cache, outputs and scores as
    eager steps, to the last bit."""
    import torch
    n, H, G, d, page, steps = 3, 8, 2, 64, 16, 20
    gen = torch.Generator().manual_seed(5)
    rows = torch.randn(steps, n, (H + 2 * G) * d, generator=gen).bfloat16().cuda()

    eager, graphed = Side(n, H, G, d, page), Side(n, H, G, d, page)
    graphed.qkv.copy_(rows[0])
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    start = [t.clone() for t in graphed.all()]
    with torch.cuda.stream(warm):
        graphed.step()
    torch.cuda.current_stream().wait_stream(warm)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.step()
    for t, s in zip(graphed.all(), start):
        t.copy_(s)
    for x in rows:
        for side in (eager, graphed):
            side.qkv.copy_(x)
        eager.step()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.all(), graphed.all()))


def test_two_loops_at_once():
    """Two decode loops on streams of their own, each with its buffers, against the same loops one after the other."""
    import torch
    n, H, G, d, page, steps = 3, 8, 2, 64, 16, 18
    gen = torch.Generator().manual_seed(6)
    rows = torch.randn(2, steps, n, (H + 2 * G) * d, generator=gen).bfloat16().cuda()
    alone, both = [[Side(n, H, G, d, page) for _ in range(2)] for _ in range(2)]
    for side, own in zip(alone, rows):
        for x in own:
            side.qkv.copy_(x)
            side.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for t in range(steps):
        for side, own, stream in zip(both, rows, streams):
            with torch.cuda.stream(stream):
                side.qkv.copy_(own[t])
                side.step()
    torch.cuda.synchronize()
    for one, other in zip(alone, both):
        assert all(torch.equal(a, b) for a, b in zip(one.all(), other.all()))
