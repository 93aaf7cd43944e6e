"""Caches in 8 bits, drafted tokens and beams over the paged key-value cache: one pass of each through its entry points.

A case names one path (``kind``), a decoder's heads and the sizes of one pass:

* ``quantise`` -- PagedCache.append into a cache of e4m3 values with a scale per row, PagedCache.read of the same rows;
* ``attention`` -- PagedCache.attention: one new token of each sequence over its whole e4m3 cache;
* ``tree`` -- PagedCache.attention_tree: the drafted tokens of each sequence over its cache and their own ancestors;
* ``keep`` -- PagedCache.keep: the accepted drafts' keys and values moved to where the sequence goes on;
* ``beam`` -- beam_select, the best continuations of each group's beams, and PagedCache.reorder by their parents.

``run`` computes them in plain torch operations, or, where ``own`` is true, through the framework.  ``exact`` restates
each in float64, sequence by sequence.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# query heads, KV heads, head dim, rotary base
SHAPES = {
    "tiny": (4, 4, 64, 1.0e4),
    "gpt2s": (12, 12, 64, 1.0e4),
    "7b": (32, 8, 128, 1.0e6),
    "8b": (32, 8, 128, 5.0e5),
}
MOST_DRAFTS = 64


def listed():
    return [
        # a decode step's new rows of a full batch, every sequence at its own length: latency
        dict(name="quantise-8b-step", kind="quantise", shape="8b", page=16, seqs=64, shortest=1, longest=2048, mix=1,
             chunk=False, bounds=True),
        # whole prompts of uneven length, 1 to 8192 rows, written and read back at once: bound by memory
        dict(name="quantise-8b-prompts", kind="quantise", shape="8b", page=64, seqs=6, shortest=1, longest=8192, mix=2,
             chunk=True, bounds=False),
        # GPT-2-small heads (a KV head for each query head), a calibration set's lengths
        dict(name="attention-gpt2s-e4m3", kind="attention", shape="gpt2s", page=32, seqs=16, shortest=1500,
             longest=2048, mix=4),
        # an uneven serving batch at the 8B heads, small pages
        dict(name="attention-8b-batch-e4m3", kind="attention", shape="8b", page=16, seqs=32, shortest=100,
             longest=8192, mix=5),
        # few rows over long caches: the length has to be split to fill the card
        dict(name="attention-8b-long-e4m3", kind="attention", shape="8b", page=64, seqs=2, shortest=20001,
             longest=32768, mix=6),
        # five drafts of one short fp32 sequence: latency alone
        dict(name="tree-tiny-f32", kind="tree", shape="tiny", dtype="f32", page=16, seqs=1, shortest=257, longest=257,
             mix=7, fewest=5, drafts=5),
        # trees of 3 to 26 drafts in a small serving batch
        dict(name="tree-8b-batch", kind="tree", shape="8b", dtype="bf16", page=16, seqs=8, shortest=500, longest=4096,
             mix=8, fewest=3, drafts=26),
        # the widest trees over long 8-bit caches: 256 query rows to a KV head, arithmetic counts
        dict(name="tree-8b-long-e4m3", kind="tree", shape="8b", dtype="e4m3", page=64, seqs=16, shortest=100,
             longest=8192, mix=9, fewest=64, drafts=64),
        # the accepted paths of a batch, the key bounds kept
        dict(name="keep-8b-batch", kind="keep", shape="8b", dtype="bf16", page=16, seqs=32, shortest=500, longest=2048,
             mix=10, fewest=3, drafts=26, bounds=True),
        # long chains of drafts at the GPT-2-small heads
        dict(name="keep-gpt2s-f32", kind="keep", shape="gpt2s", dtype="f32", page=64, seqs=8, shortest=100,
             longest=1000, mix=11, fewest=64, drafts=64, bounds=False),
        # one text, four beams, an odd vocabulary in a padded bf16 buffer
        dict(name="beam-gpt2s", kind="beam", shape="gpt2s", dtype="bf16", page=32, groups=1, beams=4, out=4, vocab=50257,
             logits="bf16", pad=2, longest=1009, mix=12),
        # a batch of texts at the largest vocabulary, fp32 logits: bound by memory
        dict(name="beam-8b-batch", kind="beam", shape="8b", dtype="bf16", page=64, groups=16, beams=8, out=8,
             vocab=128256, logits="f32", pad=0, longest=500, mix=13),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantise", "attention", "tree", "tree", "keep", "beam"])
    shape, page = rng.choice(sorted(SHAPES)), rng.choice([16, 32, 64, 128])
    case = dict(kind=kind, shape=shape, page=page, mix=rng.randrange(1 << 16))
    if kind == "beam":
        vocab, beams = _log_int(rng, 1000, 128256), _log_int(rng, 2, 16)
        return dict(case, dtype=rng.choice(["f32", "bf16"]), groups=_log_int(rng, 1, max(1, 16000000 // (vocab * beams))),
                    beams=beams, out=rng.choice([beams, beams, 2 * beams]), vocab=vocab, logits=rng.choice(["f32", "bf16"]),
                    pad=rng.choice([0, 0, 1, 7]), longest=_log_int(rng, 1, 1000))
    if kind == "quantise" and rng.random() < 0.5:
        longest = _log_int(rng, 1, 8192)
        seqs = _log_int(rng, 1, max(1, min(16, 24576 // longest)))
        chunk = True
    else:
        longest = _log_int(rng, 1, 32768 if kind == "attention" else 8192)
        seqs = _log_int(rng, 1, max(1, min(64, 64000 // longest)))
        chunk = False
    case.update(seqs=seqs, shortest=max(1, longest // rng.choice([1, 2, 16])), longest=longest)
    if kind == "quantise":
        case.update(chunk=chunk, bounds=rng.random() < 0.5)
    if kind in ("tree", "keep"):
        drafts = _log_int(rng, 1, MOST_DRAFTS)
        case.update(dtype=rng.choice(["bf16", "bf16", "f32"] + ["e4m3"] * 2 * (kind == "tree")), drafts=drafts,
                    fewest=max(1, drafts // rng.choice([1, 2, 8])), longest=max(longest, drafts),
                    shortest=max(case["shortest"], drafts))
    if kind == "keep":
        case.update(bounds=rng.random() < 0.5)
    return case


def lengths_of(case):
    """The sequences' lengths: the longest first, the others between."""
    r = random.Random(case["mix"])
    lens = [case["longest"]] + [r.randint(case["shortest"], case["longest"]) for _ in range(case["seqs"] - 1)]
    if len(lens) > 2 or (len(lens) > 1 and case.get("chunk")):
        lens[-1] = case["shortest"]
    return lens


def drafts_of(case):
    """Drafted tokens of each sequence, the last entries of it."""
    r = random.Random(case["mix"] + 1)
    return [case["drafts"]] + [r.randint(case["fewest"], case["drafts"]) for _ in range(case["seqs"] - 1)]


def parents_of(case):
    """For each sequence the parent of each draft, an earlier one, or -1 for a child of the text's last token."""
    r = random.Random(case["mix"] + 2)
    return [[r.randint(max(-1, j - 8), j - 1) for j in range(m)] for m in drafts_of(case)]


def _ancestors(parents):
    """Bit t of word j: draft t is j or an ancestor of it."""
    words = []
    for j, p in enumerate(parents):
        words.append(1 << j | (words[p] if p >= 0 else 0))
    return words


def paths_of(case):
    """For each sequence the accepted drafts: the way from the root to one of them."""
    r = random.Random(case["mix"] + 3)
    paths = []
    for parents in parents_of(case):
        word = _ancestors(parents)[r.randrange(len(parents))]
        paths.append([t for t in range(len(parents)) if word >> t & 1])
    return paths


def _width(dtype):
    return {"f32": 4, "bf16": 2, "e4m3": 1}[dtype]


def work(case):
    H, G, d, _ = SHAPES[case["shape"]]
    page = case["page"]
    if case["kind"] == "beam":
        rows = case["groups"] * case["beams"]
        read = rows * case["vocab"]
        rest = case["longest"] % page
        # the page in progress of each beam, read and written; a table
        moved = 2 * rows * rest * G * 2 * d * _width(case["dtype"]) + 2 * 4 * rows * (case["longest"] // page + 2)
        return {"bytes": read * _width(case["logits"]) + moved + case["groups"] * case["out"] * 12, "flops": 3 * read}
    lens = lengths_of(case)
    if case["kind"] == "quantise":
        rows = sum(lens) if case["chunk"] else len(lens)
        data = 2 * rows * H * d * 2 + rows * G * (2 * d * (2 + 1 + 1 + 2) + 4) + 8 * rows
        if case["bounds"]:
            touched = sum((n + page - 1) // page for n in lens) if case["chunk"] else len(lens)
            data += touched * G * 2 * d * 2 * (1 if case["chunk"] else 2)
        return {"bytes": data, "flops": 3 * rows * (H + G) * d + 8 * rows * G * d}
    if case["kind"] == "attention":
        n = len(lens)
        return {"bytes": sum(lens) * G * 2 * (d + 1) + 2 * n * H * d * 2 + 4 * n * H, "flops": 4 * sum(lens) * H * d}
    drafts = drafts_of(case)
    if case["kind"] == "tree":
        es, wide = _width(case["dtype"]), 4 if case["dtype"] == "f32" else 2
        row = d * es + (case["dtype"] == "e4m3")
        return {"bytes": sum(lens) * G * 2 * row + sum(drafts) * (2 * H * d * wide + 4 * H + 8),
                "flops": 4 * sum(n * m for n, m in zip(lens, drafts)) * H * d}
    moved = sum(len(p) for p in paths_of(case))
    data = 4 * moved * G * d * _width(case["dtype"]) + 4 * moved
    if case["bounds"]:
        data += len(lens) * G * 4 * d * _width(case["dtype"])
    return {"bytes": data, "flops": 2 * moved * G * d}


def _torch_type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.bfloat16}[name]


def _power(e):
    """2^e in float32 of whole numbers -126 .. 127, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_e4m3(x):
    """Codes and scales (as powers of two) of rows x [..., d]: the largest value of a row at 448 times its scale at most."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))
    e = (e - 9 + (m > 0.875)).clamp(-117, 120)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _from_e4m3(codes, scales):
    """The float32 values of codes [..., d] with scales [...]."""
    return codes.float() * _power(scales.to(torch.int32) - 127)[..., None]


def _tables(case, lens, g, dev):
    """Pages in the order in which a running server hands them out: any."""
    page = case["page"]
    counts = [(x + page - 1) // page for x in lens]
    order = torch.randperm(sum(counts) + 8, generator=g, device=dev).to(torch.int32)
    pages = torch.full((len(lens), max(counts)), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, c in enumerate(counts):
        pages[i, :c] = order[at:at + c]
        at += c
    return pages, sum(counts) + 8


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = torch.device("cuda")
    H, G, d, theta = SHAPES[case["shape"]]
    page = case["page"]
    state = dict(case=case)
    if case["kind"] == "beam":
        groups, beams, vocab, length = case["groups"], case["beams"], case["vocab"], case["longest"]
        rows, full = groups * beams, length // page
        # the logits of a language model: a bulk, and a few likely tokens of each row far above it
        x = torch.randn(rows, vocab + case["pad"], generator=g, device=dev).mul_(2.0)
        likely = torch.randint(0, vocab, (rows, 24), generator=g, device=dev)
        x.scatter_add_(1, likely, torch.rand(rows, 24, generator=g, device=dev) * 12.0)
        state["logits"] = x.to(_torch_type(case["logits"]))[:, :vocab]
        state["scores"] = -10.0 * torch.rand(groups, beams, generator=g, device=dev).sort(dim=1).values
        # every eighth text or so is at its first step: one beam holds it, the others wait
        first = torch.rand(groups, 1, generator=g, device=dev) < 0.125
        state["scores"].masked_fill_(first & (torch.arange(beams, device=dev) > 0), -math.inf)
        state["ended"] = (torch.rand(groups, beams, generator=g, device=dev) < 0.1) & ~first
        state["end_token"] = vocab - 1
        # a group's full pages are those of its common beginning, then each beam's own
        shared, pages_each = max(0, full - 2), full - max(0, full - 2) + 2
        n_pages = groups * (shared + beams * pages_each) + 8
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        common = order[:groups * shared].view(groups, 1, shared).expand(-1, beams, -1)
        apart = order[groups * shared:n_pages - 8].view(groups, beams, pages_each)
        state["pages"] = torch.cat([common, apart], 2).reshape(rows, -1).contiguous()
        lens = [length] * rows
        state["parents"] = torch.empty(groups, case["out"], dtype=torch.int32, device=dev)
        state["tokens"] = torch.empty_like(state["parents"])
        state["best"] = torch.empty(groups, case["out"], device=dev)
        state["new_pages"] = torch.empty_like(state["pages"])
    else:
        lens = lengths_of(case)
        state["pages"], n_pages = _tables(case, lens, g, dev)
    n = len(lens)
    state["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    # keys have a common part in each channel, and a few channels are large
    mean = torch.randn(G, 1, d, generator=g, device=dev)
    wide = 1.0 + 4.0 * (torch.rand(G, 1, d, generator=g, device=dev) > 0.95)
    k = torch.randn(n_pages, G, page, d, generator=g, device=dev).mul_(wide).add_(mean)
    v = torch.randn(n_pages, G, page, d, generator=g, device=dev)
    dtype = case.get("dtype", "e4m3")
    if dtype == "e4m3":
        state["k"], state["k_scales"] = _to_e4m3(k)
        state["v"], state["v_scales"] = _to_e4m3(v)
    else:
        state["k"], state["v"] = k.to(_torch_type(dtype)), v.to(_torch_type(dtype))
    if case.get("bounds"):
        seen = _from_e4m3(state["k"], state["k_scales"]) if dtype == "e4m3" else state["k"]
        state["bounds"] = torch.stack([seen.amin(2), seen.amax(2)], 2).to(_torch_type(dtype))
    del k, v
    if case["kind"] == "quantise":
        rows = sum(lens) if case["chunk"] else n
        # a row of the fused projection: queries, keys, values
        qkv = torch.randn(rows, (H + 2 * G) * d, generator=g, device=dev)
        qkv[:, H * d:(H + G) * d].view(rows, G, d).mul_(wide[:, 0]).add_(mean[:, 0])
        qkv = qkv.to(torch.bfloat16)
        state["q"] = qkv[:, :H * d].view(rows, H, d)
        state["new_k"] = qkv[:, H * d:(H + G) * d].view(rows, G, d)
        state["new_v"] = qkv[:, (H + G) * d:].view(rows, G, d)
        state["q_out"] = torch.empty(rows, H, d, dtype=torch.bfloat16, device=dev)
        state["k_out"] = torch.empty(rows, G, d, dtype=torch.bfloat16, device=dev)
        state["v_out"] = torch.empty_like(state["k_out"])
        offsets, last = [0], torch.tensor(lens, device=dev)
        for x in lens:
            offsets.append(offsets[-1] + (x if case["chunk"] else 1))
        state["offsets"], state["theta"] = offsets if case["chunk"] else None, theta
        # a compressed cache is shorter than the text: positions run ahead of the entries by what was dropped
        dropped = torch.randint(0, 4 * max(lens), (n,), generator=g, device=dev)
        counts = last if case["chunk"] else torch.ones_like(last)
        owner = torch.repeat_interleave(torch.arange(n, device=dev), counts)
        within = torch.arange(rows, device=dev) - (torch.cumsum(counts, 0) - counts)[owner]
        state["owner"], state["entry"] = owner, last[owner] - counts[owner] + within
        state["positions"] = (state["entry"] + dropped[owner]).to(torch.int32)
    elif case["kind"] == "attention":
        state["q"] = torch.randn(n, H, d, generator=g, device=dev).mul_(2.0).to(torch.bfloat16)
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(n, H, device=dev)
    elif case["kind"] in ("tree", "keep"):
        drafts = drafts_of(case)
        state["offsets"] = [0]
        for m in drafts:
            state["offsets"].append(state["offsets"][-1] + m)
        if case["kind"] == "tree":
            rows = sum(drafts)
            words = [w - (1 << 64) if w >> 63 else w for p in parents_of(case) for w in _ancestors(p)]
            state["masks"] = torch.tensor(words, dtype=torch.int64, device=dev)
            state["drafts"] = torch.tensor(drafts, device=dev)
            state["q"] = torch.randn(rows, H, d, generator=g, device=dev).mul_(2.0).to(_torch_type(dtype))
            state["out"] = torch.empty_like(state["q"])
            state["lse"] = torch.empty(rows, H, device=dev)
        else:
            paths = paths_of(case)
            kept = torch.full((n, max(drafts)), -1, dtype=torch.int32)
            for i, p in enumerate(paths):
                kept[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
            state["kept"], state["drafts"] = kept.to(dev), torch.tensor(drafts, device=dev)
    return state


# ----------------------------------------------------------------------------- the framework's calls

def _workspace(state, size):
    """The caller's workspace: allocated once, kept as a serving loop keeps it."""
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(size(), 1), dtype=torch.uint8, device="cuda")
    return state["workspace"]


def _framework(state):
    import paper_2608_08684_amd as rk

    case = state["case"]
    if "cache" not in state:   # the handles that a serving loop keeps
        state["cache"] = rk.PagedCache(state["k"], state["v"], state.get("bounds"), k_scales=state.get("k_scales"),
                                       v_scales=state.get("v_scales"))
        state["seqs"] = rk.PagedSeqs(state["pages"], state["lengths"])
    cache, seqs = state["cache"], state["seqs"]
    if case["kind"] == "quantise":
        cache.append(seqs, state["new_k"], state["new_v"], row_offsets=state["offsets"], q=state["q"],
                     q_out=state["q_out"], positions=state["positions"], rope_theta=state["theta"])
        cache.read(seqs, state["k_out"], state["v_out"], row_offsets=state["offsets"])
        out = {"k": state["k_out"], "v": state["v_out"], "q": state["q_out"]}
        return dict(out, bounds=state["bounds"]) if case["bounds"] else out
    if case["kind"] == "keep":
        cache.keep(seqs, state["offsets"], state["kept"])
        out = {"k": state["k"], "v": state["v"]}
        return dict(out, bounds=state["bounds"]) if case["bounds"] else out
    if case["kind"] == "beam":
        groups, beams, vocab, n_out = case["groups"], case["beams"], case["vocab"], case["out"]
        ws = _workspace(state, lambda: rk.beam_select_workspace_size(groups, beams, vocab, n_out, case["logits"]))
        rk.beam_select(state["logits"], state["scores"], state["parents"], state["tokens"], state["best"], ws,
                       ended=state["ended"], end_token=state["end_token"])
        parents = state["parents"] if n_out == beams else state["parents"][:, :beams].contiguous()
        cache.reorder(seqs, parents, pages_out=state["new_pages"])
        return {"parents": state["parents"], "tokens": state["tokens"], "scores": state["best"],
                "pages": state["new_pages"], "k": state["k"], "v": state["v"]}
    n_heads = state["q"].shape[1]
    if case["kind"] == "attention":
        ws = _workspace(state, lambda: cache.workspace_size(seqs.n_seqs, seqs.max_pages, n_heads))
        cache.attention(seqs, state["q"], state["out"], ws, lse=state["lse"])
    else:
        ws = _workspace(state, lambda: cache.tree_workspace_size(seqs.n_seqs, len(state["q"]), seqs.max_pages, n_heads))
        cache.attention_tree(seqs, state["q"], state["out"], ws, state["offsets"], masks=state["masks"],
                             lse=state["lse"])
    return {"out": state["out"], "lse": state["lse"]}


# ----------------------------------------------------------------------------- plain forms

def _rotate(x, positions, theta):
    """Rotate-half rotary embedding of x [rows, heads, d] in float32; the angles in 64 bits."""
    half = x.shape[-1] // 2
    freq = theta ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    angle = positions.to(torch.float64)[:, None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _bounds_with(bounds, page, fresh, keys):
    """Each page's bounds with new keys [rows, KV heads, d]; those of the fresh pages begin anew."""
    wide = page[:, None, None].expand(-1, *keys.shape[1:])
    lo, hi = bounds[:, :, 0].float(), bounds[:, :, 1].float()
    lo[fresh], hi[fresh] = math.inf, -math.inf
    lo.scatter_reduce_(0, wide, keys.float(), "amin")
    hi.scatter_reduce_(0, wide, keys.float(), "amax")
    bounds.copy_(torch.stack([lo, hi], 2).to(bounds.dtype))


def _quantise(state):
    page, owner, entry = state["case"]["page"], state["owner"], state["entry"]
    at, slot = state["pages"][owner, entry // page].long(), entry % page
    k, k_scales = _to_e4m3(_rotate(state["new_k"], state["positions"], state["theta"]))
    v, v_scales = _to_e4m3(state["new_v"])
    held_k, held_v = state["k"].view(torch.uint8), state["v"].view(torch.uint8)
    held_k[at, :, slot], held_v[at, :, slot] = k.view(torch.uint8), v.view(torch.uint8)
    state["k_scales"][at, :, slot], state["v_scales"][at, :, slot] = k_scales, v_scales
    out = {"q": _rotate(state["q"], state["positions"], state["theta"]).to(torch.bfloat16)}
    if "bounds" in state:
        _bounds_with(state["bounds"], at, at[slot == 0], _from_e4m3(k, k_scales))
        out["bounds"] = state["bounds"]
    out["k"] = _from_e4m3(held_k[at, :, slot].view(torch.float8_e4m3fn), state["k_scales"][at, :, slot]).to(torch.bfloat16)
    out["v"] = _from_e4m3(held_v[at, :, slot].view(torch.float8_e4m3fn), state["v_scales"][at, :, slot]).to(torch.bfloat16)
    return out


def _entries(state, name):
    """All keys or values of the sequences in float32 [n, KV heads, entries, d]."""
    pages = state["pages"].clamp(min=0).long()
    x = state[name]
    if x.dtype == torch.float8_e4m3fn:
        x = _from_e4m3(x.view(torch.uint8)[pages].view(x.dtype), state[name + "_scales"][pages])
    else:
        x = x[pages].float()
    n, width, G, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, G, width * page, d)


def _attend(state, q, see):
    """Attention of q [n, rows, H, d] over the entries that ``see`` [n, rows, entries] lets through."""
    n, rows, H, d = q.shape
    keys = _entries(state, "k")
    G = keys.shape[1]
    q = q.float().view(n, rows, G, H // G, d).permute(0, 2, 1, 3, 4).reshape(n, G, rows * (H // G), d)
    s = torch.matmul(q, keys.transpose(2, 3).contiguous()).view(n, G, rows, H // G, -1)
    del keys
    s = s.div_(math.sqrt(d)).masked_fill_(~see[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = s.sub_(m.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = e.sum(-1, keepdim=True)
    out = torch.matmul((e / total.clamp(min=1e-30)).view(n, G, rows * (H // G), -1), _entries(state, "v"))
    out = out.view(n, G, rows, H // G, d).permute(0, 2, 1, 3, 4).reshape(n, rows, H, d)
    lse = (m + total.log()).permute(0, 2, 1, 3, 4).reshape(n, rows, H)
    return out.to(state["q"].dtype), lse


def _attention(state):
    entries = state["pages"].shape[1] * state["case"]["page"]
    see = torch.arange(entries, device=state["pages"].device) < state["lengths"][:, None]
    out, lse = _attend(state, state["q"][:, None], see[:, None])
    return {"out": out[:, 0], "lse": lse[:, 0]}


def _tree(state):
    drafts, n, most = state["drafts"], len(state["lengths"]), state["case"]["drafts"]
    dev = drafts.device
    at = torch.arange(most, device=dev)
    row = (torch.cumsum(drafts, 0) - drafts)[:, None] + at.clamp(max=most - 1)
    real = at < drafts[:, None]
    row = torch.where(real, row, 0)
    words = state["masks"][row]                                     # [n, most]
    u = torch.arange(state["pages"].shape[1] * state["case"]["page"], device=dev)
    t = (u - (state["lengths"] - drafts)[:, None])[:, None]          # [n, 1, entries]: which draft an entry is
    see = (t < 0) | ((words[:, :, None] >> t.clamp(0, 63) & 1).bool() & (t < drafts[:, None, None]))
    out, lse = _attend(state, state["q"][row], see)
    return {"out": out[real], "lse": lse[real]}


def _keep(state):
    page, kept = state["case"]["page"], state["kept"].long()
    seq, j = torch.nonzero(kept >= 0, as_tuple=True)
    base = state["lengths"] - state["drafts"]
    old, new = base[seq] + kept[seq, j], base[seq] + j
    src, dst = (state["pages"][seq, e // page].long() for e in (old, new))
    keys, values = state["k"][src, :, old % page], state["v"][src, :, old % page]
    state["k"][dst, :, new % page], state["v"][dst, :, new % page] = keys, values
    out = {"k": state["k"], "v": state["v"]}
    if "bounds" in state:
        _bounds_with(state["bounds"], dst, dst[new % page == 0], keys)
        out["bounds"] = state["bounds"]
    return out


def _beam(state):
    case = state["case"]
    groups, beams, n_out = case["groups"], case["beams"], case["out"]
    x = state["logits"].float()
    # one whole number that orders a row by logit, then by lower token
    ids = torch.arange(x.shape[1], device=x.device)
    bits = (x + 0.0).view(torch.int32).long()
    key = (torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) << 32) | (0x7FFFFFFF - ids)
    token = 0x7FFFFFFF - (key.topk(min(n_out, x.shape[1]), dim=-1).values & 0x7FFFFFFF)
    del key, bits
    # scores between beams in 64 bits: whole numbers hang on their order
    m = x.amax(-1, keepdim=True)
    total = (x - m).double().exp().sum(-1, keepdim=True)
    logp = x.gather(1, token).double() - m.double() - total.log()
    ended = state["ended"].view(-1, 1)
    first = torch.arange(token.shape[1], device=x.device) == 0
    token = torch.where(ended, state["end_token"], token)
    logp = torch.where(ended, torch.where(first, 0.0, -math.inf), logp)
    score = (state["scores"].double().view(-1, 1) + logp).view(groups, -1)
    best = score.sort(dim=1, descending=True, stable=True)
    pick, value = best.indices[:, :n_out], best.values[:, :n_out].float()
    there = value > -math.inf
    parents = torch.where(there, pick // token.shape[1], -1).to(torch.int32)
    tokens = torch.where(there, token.view(groups, -1).gather(1, pick), -1).to(torch.int32)
    # the caches follow: full pages by the table, the page in progress by its entries
    page, length = case["page"], case["longest"]
    full, rest = length // page, length % page
    own_row = torch.arange(groups * beams, device=x.device).view(groups, beams)
    new = parents[:, :beams].long()
    source = torch.where(new >= 0, new + own_row[:, :1], own_row).view(-1)
    pages = state["pages"].clone()
    pages[:, :full] = state["pages"][source, :full]
    if rest:
        src, dst = state["pages"][source, full].long(), state["pages"][:, full].long()
        state["k"][dst, :, :rest], state["v"][dst, :, :rest] = state["k"][src, :, :rest], state["v"][src, :, :rest]
    return {"parents": parents, "tokens": tokens, "scores": value, "pages": pages, "k": state["k"], "v": state["v"]}


def run(state):
    if own:
        return _framework(state)
    return {"quantise": _quantise, "attention": _attention, "tree": _tree, "keep": _keep, "beam": _beam}[
        state["case"]["kind"]](state)


# ----------------------------------------------------------------------------- float64 restatement

def _turned(x, position, theta):
    d = x.shape[-1]
    x = x.double()
    out = torch.empty_like(x)
    for j in range(d // 2):
        angle = position.double() * math.exp(-2.0 * j / d * math.log(theta))
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        out[..., j] = x[..., j] * c - x[..., j + d // 2] * s
        out[..., j + d // 2] = x[..., j + d // 2] * c + x[..., j] * s
    return out


def _rounded(x):
    """Float64 rows rounded to 4 significant bits of a number of at least 2^-6, below that to whole steps of 2^-9, in
    units of the power of two at which no value of the row exceeds 448."""
    unit = torch.ones_like(x[..., :1])
    top = x.abs().amax(-1, keepdim=True)
    while bool((top > 448.0 * unit).any()):
        unit = torch.where(top > 448.0 * unit, unit * 2, unit)
    while bool(((top <= 224.0 * unit) & (unit > 2.0 ** -117)).any()):
        unit = torch.where((top <= 224.0 * unit) & (unit > 2.0 ** -117), unit / 2, unit)
    y = x / unit
    bits = torch.frexp(y.abs().clamp(min=2.0 ** -6))[1].long() - 4   # of a step: a value has 4 bits
    step = (bits + 1023 << 52).view(torch.float64)
    return torch.round(y / step) * step * unit


def _held(state, name, pages, h):
    """One head's keys or values of the given pages in float64 [pages * page size, d]."""
    x = state[name]
    if x.dtype == torch.float8_e4m3fn:
        scale = (state[name + "_scales"][pages, h].long() - 127 + 1023 << 52).view(torch.float64)
        got = x.view(torch.uint8)[pages, h].view(x.dtype).float().double() * scale[..., None]
    else:
        got = x[pages, h].double()
    return got.reshape(-1, x.shape[-1])


def _exact_moves(state, moves):
    """The whole caches in float64 after moves (page, slot) <- (page, slot), all read before any is written."""
    out = {}
    for name in ("k", "v"):
        old = state[name].double()
        new = old.clone()
        for (p, s), (q, t) in moves:
            new[p, :, s] = old[q, :, t]
        out[name] = new
    return out


def exact(case, seed):
    state = prepare(case, seed)
    page = case["page"]
    table = state["pages"].cpu()
    if case["kind"] == "beam":
        groups, beams, n_out = case["groups"], case["beams"], case["out"]
        best, parents = [], []
        for i in range(groups):
            scores = []
            for b in range(beams):
                if bool(state["ended"][i, b]):
                    row = torch.full((case["vocab"],), -math.inf, dtype=torch.float64, device="cuda")
                    row[state["end_token"]] = 0.0
                else:
                    row = torch.log_softmax(state["logits"][i * beams + b].double(), 0)
                scores.append(row + state["scores"][i, b].double())
            scores = torch.stack(scores)
            values, at = torch.topk(scores.view(-1), n_out)
            best.append(values)
            parents.append([int(p) if math.isfinite(s) else b for b, (p, s) in
                            enumerate(zip((at // case["vocab"]).tolist(), values.tolist()))][:beams])
        full, rest = case["longest"] // page, case["longest"] % page
        moves = [((int(table[i * beams + b, full]), s), (int(table[i * beams + p, full]), s))
                 for i in range(groups) for b, p in enumerate(parents[i]) if b != p for s in range(rest)]
        return dict(_exact_moves(state, moves), parents=None, tokens=None, pages=None, scores=torch.stack(best))
    lens = lengths_of(case)
    if case["kind"] == "keep":
        moves = []
        for i, (length, m, path) in enumerate(zip(lens, drafts_of(case), paths_of(case))):
            for j, t in enumerate(path):
                a, b = length - m + j, length - m + t
                moves.append(((int(table[i, a // page]), a % page), (int(table[i, b // page]), b % page)))
        out = _exact_moves(state, moves)
        if case["bounds"]:
            b = state["bounds"].double()
            for (p, s), _ in moves:
                key = out["k"][p, :, s]
                b[p, :, 0] = key if s == 0 else torch.minimum(key, b[p, :, 0])
                b[p, :, 1] = key if s == 0 else torch.maximum(key, b[p, :, 1])
            out["bounds"] = b
        return out
    if case["kind"] == "quantise":
        k = _rounded(_turned(state["new_k"], state["positions"], state["theta"]))
        out = {"k": k, "v": _rounded(state["new_v"].double()),
               "q": _turned(state["q"], state["positions"], state["theta"])}
        if case["bounds"]:
            b, row = state["bounds"].double(), 0
            for i, length in enumerate(lens):
                e = 0 if case["chunk"] else length - 1
                while e < length:
                    p, c = int(table[i, e // page]), min(page - e % page, length - e)
                    lo, hi = k[row:row + c].amin(0), k[row:row + c].amax(0)
                    b[p, :, 0] = lo if e % page == 0 else torch.minimum(lo, b[p, :, 0])
                    b[p, :, 1] = hi if e % page == 0 else torch.maximum(hi, b[p, :, 1])
                    e, row = e + c, row + c
            out["bounds"] = b
        return out
    H, G, d, _ = SHAPES[case["shape"]]
    drafts = drafts_of(case) if case["kind"] == "tree" else [1] * len(lens)
    trees = parents_of(case) if case["kind"] == "tree" else [[-1]] * len(lens)
    outs, lses, row = [], [], 0
    for i, (length, m, parents) in enumerate(zip(lens, drafts, trees)):
        mine = state["pages"][i, :(length + page - 1) // page].long()
        see = torch.ones(m, length, dtype=torch.bool)
        for j in range(m):
            see[j, length - m:] = False
            t = j
            while t >= 0:
                see[j, length - m + t] = True
                t = parents[t]
        see = see.cuda()
        out = torch.empty(m, H, d, dtype=torch.float64, device="cuda")
        lse = torch.empty(m, H, dtype=torch.float64, device="cuda")
        for h in range(H):
            k, v = (_held(state, name, mine, h // (H // G))[:length] for name in ("k", "v"))
            s = state["q"][row:row + m, h].double() @ k.T / math.sqrt(d)
            s = s.masked_fill(~see, -math.inf)
            lse[:, h] = torch.logsumexp(s, 1)
            out[:, h] = (s - lse[:, h, None]).exp() @ v
        outs.append(out)
        lses.append(lse)
        row += m
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
