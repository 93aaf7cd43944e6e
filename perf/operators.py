"""The serving operators over a paged key-value cache, one pass of each through its public entry point.

A case names one operator (``kind``), a decoder's heads and the sizes of one call:

* ``append``    -- PagedCache.append: new keys and values into the pages of their sequences, keys and queries rotated;
* ``attention`` -- PagedCache.attention: one new token of each sequence over its whole cache;
* ``selected``  -- PagedCache.attention_selected: the same over the pages that the key bounds rank highest;
* ``logprobs``  -- token_logprobs: log probability and rank of given tokens, entropy and the best alternatives.

``run`` computes them in plain torch operations, or, where ``own`` is true, through the framework.  ``exact`` restates
each in float64, sequence by sequence.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# query heads, KV heads, head dim, rotary base, dtype
SHAPES = {
    "tiny-f32": (4, 4, 64, 1.0e4, "f32"),
    "gpt2s": (12, 12, 64, 1.0e4, "bf16"),
    "gpt2s-f32": (12, 12, 64, 1.0e4, "f32"),
    "7b": (32, 8, 128, 1.0e6, "bf16"),
    "8b": (32, 8, 128, 5.0e5, "bf16"),
}


def listed():
    return [
        # one token of one sequence into the smallest model's fp32 cache: latency alone
        dict(name="append-tiny-f32", kind="append", shape="tiny-f32", page=16, seqs=1, shortest=257, longest=257, mix=0,
             chunk=False, bounds=True),
        # a decode step's new rows of a full batch, every sequence at its own length
        dict(name="append-8b-step", kind="append", shape="8b", page=16, seqs=64, shortest=1, longest=2048, mix=1,
             chunk=False, bounds=True),
        # whole prompts of uneven length, 1 to 8192 rows, written at once: bound by memory
        dict(name="append-8b-prompts", kind="append", shape="8b", page=64, seqs=6, shortest=1, longest=8192, mix=2,
             chunk=True, bounds=True),
        # a few short fp32 caches, one of a single token: the check against the bf16 path
        dict(name="attention-tiny-f32", kind="attention", shape="tiny-f32", page=16, seqs=3, shortest=1, longest=257,
             mix=3),
        # GPT-2-small heads (a KV head for each query head), a calibration set's lengths
        dict(name="attention-gpt2s", kind="attention", shape="gpt2s", page=32, seqs=16, shortest=1500, longest=2048,
             mix=4),
        # an uneven serving batch at the 8B heads, small pages
        dict(name="attention-8b-batch", kind="attention", shape="8b", page=16, seqs=32, shortest=100, longest=8192,
             mix=5),
        # few rows over long caches: the length has to be split to fill the card
        dict(name="attention-8b-long", kind="attention", shape="8b", page=64, seqs=2, shortest=20001, longest=32768,
             mix=6),
        # a fifth of a short cache, in small pages: four dependent steps, latency counts
        dict(name="selected-gpt2s", kind="selected", shape="gpt2s", page=16, seqs=8, shortest=1500, longest=2048, mix=7,
             select=26, first=1, last=2),
        # an eighth of long caches
        dict(name="selected-8b-long", kind="selected", shape="8b", page=64, seqs=4, shortest=20001, longest=32768, mix=8,
             select=64, first=1, last=2),
        # the logits of one decode step of a batch, with five alternatives
        dict(name="logprobs-step", kind="logprobs", dtype="f32", rows=16, vocab=32000, pad=0, top=5),
        # bf16 logits of an odd vocabulary in a padded buffer: rows start at any 2-byte address
        dict(name="logprobs-odd-bf16", kind="logprobs", dtype="bf16", rows=301, vocab=50257, pad=2, top=20),
        # an evaluation window at the largest vocabulary, fp32: bound by memory
        dict(name="logprobs-8b-window", kind="logprobs", dtype="f32", rows=1024, vocab=128256, pad=0, top=20),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "selected", "selected", "logprobs"])
    if kind == "logprobs":
        vocab = _log_int(rng, 1000, 128256)
        rows = _log_int(rng, 1, max(1, min(2048, 100000000 // vocab)))
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 7]),
                    top=rng.choice([0, 1, 5, 20, 32]))
    shape = rng.choice(sorted(SHAPES))
    page = rng.choice([16, 32, 64, 128])
    if kind == "append" and rng.random() < 0.5:
        longest = _log_int(rng, 1, 8192)
        seqs = _log_int(rng, 1, max(1, min(16, 24576 // longest)))
        chunk = True
    else:
        longest = _log_int(rng, 1 if kind != "selected" else 600, 32768)
        seqs = _log_int(rng, 1, max(1, min(64, 94000 // longest)))
        chunk = False
    case = dict(kind=kind, shape=shape, page=page, seqs=seqs, shortest=max(1, longest // rng.choice([1, 2, 16])),
                longest=longest, mix=rng.randrange(1 << 16))
    if kind == "append":
        case.update(chunk=chunk, bounds=rng.random() < 0.7)
    if kind == "selected":
        first, last = rng.choice([0, 1, 2]), rng.choice([1, 2, 4])
        case.update(select=max(first + last, _log_int(rng, 4, max(4, longest // page // 4))), first=first, last=last)
    return case


def lengths_of(case):
    """The sequences' lengths: the longest first, the others between."""
    r = random.Random(case["mix"])
    lens = [case["longest"]] + [r.randint(case["shortest"], case["longest"]) for _ in range(case["seqs"] - 1)]
    if case["kind"] == "append" and case["chunk"] and len(lens) > 1:
        lens[-1] = case["shortest"]
    if case["kind"] == "attention" and case["seqs"] > 2:
        lens[1] = case["shortest"]
    return lens


def _width(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    if case["kind"] == "logprobs":
        n, out = case["rows"] * case["vocab"], case["rows"] * (16 + 8 * case["top"])
        return {"bytes": n * _width(case["dtype"]) + out, "flops": 5 * n}
    H, G, d, _, dtype = SHAPES[case["shape"]]
    es, lens, page = _width(dtype), lengths_of(case), case["page"]
    if case["kind"] == "append":
        rows = sum(lens) if case["chunk"] else len(lens)
        data = 2 * rows * (H + 2 * G) * d * es + 8 * rows
        touched = sum((n + page - 1) // page for n in lens) if case["chunk"] else len(lens)
        if case["bounds"]:   # a step's bounds are read and written, a new page's only written
            data += touched * G * 2 * d * es * (1 if case["chunk"] else 2)
        return {"bytes": data, "flops": 3 * rows * (H + G) * d}
    read = lens
    extra = 0
    if case["kind"] == "selected":
        n_pages = [(n + page - 1) // page for n in lens]
        extra = sum(n_pages) * G * 2 * d * es
        read = [n if p <= case["select"] else case["select"] * page - (p * page - n) for n, p in zip(lens, n_pages)]
        extra += 4 * len(lens) * G * case["select"]
    keys = sum(read)
    return {"bytes": 2 * keys * G * d * es + extra + 2 * len(lens) * H * d * es + 4 * len(lens) * H,
            "flops": 4 * keys * H * d + (4 * sum(lens) // page * G * d if case["kind"] == "selected" else 0)}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _generator(seed)
    dev = torch.device("cuda")
    if case["kind"] == "logprobs":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        rows, vocab, top = case["rows"], case["vocab"], case["top"]
        # the logits of a language model: a bulk, and a few likely tokens of each row far above it
        x = torch.randn(rows, vocab + case["pad"], generator=g, device=dev).mul_(2.0)
        likely = torch.randint(0, vocab, (rows, 24), generator=g, device=dev)
        x.scatter_add_(1, likely, torch.rand(rows, 24, generator=g, device=dev) * 12.0)
        pick = torch.randint(0, 24, (rows, 1), generator=g, device=dev)
        return dict(case=case, logits=x.to(dtype)[:, :vocab], tokens=likely.gather(1, pick)[:, 0].to(torch.int32),
                    logprob=torch.empty(rows, device=dev), entropy=torch.empty(rows, device=dev),
                    rank=torch.empty(rows, dtype=torch.int32, device=dev),
                    top_ids=torch.empty(rows, top, dtype=torch.int32, device=dev),
                    top_logprobs=torch.empty(rows, top, device=dev))
    H, G, d, theta, name = SHAPES[case["shape"]]
    dtype = torch.bfloat16 if name == "bf16" else torch.float32
    page, lens = case["page"], lengths_of(case)
    n, width = len(lens), (max(lens) + page - 1) // page
    used = sum((x + page - 1) // page for x in lens)
    n_pages = used + 8
    # pages in the order in which a running server hands them out: any
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    pages = torch.full((n, width), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, x in enumerate(lens):
        c = (x + page - 1) // page
        pages[i, :c] = order[at:at + c]
        at += c
    # keys have a common part in each channel, and a few channels are large
    mean = torch.randn(G, 1, d, generator=g, device=dev)
    wide = 1.0 + 4.0 * (torch.rand(G, 1, d, generator=g, device=dev) > 0.95)
    k = torch.randn(n_pages, G, page, d, generator=g, device=dev).mul_(wide).add_(mean).to(dtype)
    v = torch.randn(n_pages, G, page, d, generator=g, device=dev).to(dtype)
    state = dict(case=case, k=k, v=v, pages=pages, lengths=torch.tensor(lens, dtype=torch.int32, device=dev))
    if case["kind"] == "append":
        rows = sum(lens) if case["chunk"] else n
        # a row of the fused projection: queries, keys, values
        qkv = torch.randn(rows, (H + 2 * G) * d, generator=g, device=dev).to(dtype)
        state["q"] = qkv[:, :H * d].view(rows, H, d)
        state["new_k"] = qkv[:, H * d:(H + G) * d].view(rows, G, d)
        state["new_v"] = qkv[:, (H + G) * d:].view(rows, G, d)
        state["q_out"] = torch.empty(rows, H, d, dtype=dtype, device=dev)
        offsets, last = [0], torch.tensor(lens, device=dev)
        for x in lens:
            offsets.append(offsets[-1] + (x if case["chunk"] else 1))
        state["offsets"] = offsets if case["chunk"] else None
        state["theta"] = theta
        # a compressed cache is shorter than the text: positions run ahead of the entries by what was dropped
        dropped = torch.randint(0, 4 * max(lens), (n,), generator=g, device=dev)
        counts = last if case["chunk"] else torch.ones_like(last)
        owner = torch.repeat_interleave(torch.arange(n, device=dev), counts)
        within = torch.arange(rows, device=dev) - (torch.cumsum(counts, 0) - counts)[owner]
        state["positions"] = (last[owner] - counts[owner] + within + dropped[owner]).to(torch.int32)
        state["owner"], state["entry"] = owner, last[owner] - counts[owner] + within
        if case["bounds"]:
            state["bounds"] = torch.stack([k.amin(2), k.amax(2)], 2)
        return state
    state["q"] = torch.randn(n, H, d, generator=g, device=dev).mul_(2.0).to(dtype)
    state["out"] = torch.empty(n, H, d, dtype=dtype, device=dev)
    state["lse"] = torch.empty(n, H, device=dev)
    if case["kind"] == "selected":
        state["bounds"] = torch.stack([k.amin(2), k.amax(2)], 2)
        state["chosen"] = torch.empty(n, G, case["select"], dtype=torch.int32, device=dev)
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
    if case["kind"] == "logprobs":
        rows, top = case["rows"], case["top"]
        ws = _workspace(state, lambda: rk.token_logprobs_workspace_size(rows, case["vocab"], top, case["dtype"]))
        rk.token_logprobs(state["logits"], state["tokens"], ws, logprob=state["logprob"], rank=state["rank"],
                          entropy=state["entropy"], top_ids=state["top_ids"] if top else None,
                          top_logprobs=state["top_logprobs"] if top else None)
        return {key: state[key] for key in ("logprob", "rank", "entropy", "top_ids", "top_logprobs")}
    if "cache" not in state:   # the handles that a serving loop keeps
        state["cache"] = rk.PagedCache(state["k"], state["v"], state.get("bounds"))
        state["seqs"] = rk.PagedSeqs(state["pages"], state["lengths"])
    cache, seqs = state["cache"], state["seqs"]
    if case["kind"] == "append":
        cache.append(seqs, state["new_k"], state["new_v"], row_offsets=state["offsets"], q=state["q"],
                     q_out=state["q_out"], positions=state["positions"], rope_theta=state["theta"])
        out = {"k": state["k"], "v": state["v"], "q": state["q_out"]}
        if case["bounds"]:
            out["bounds"] = state["bounds"]
        return out
    select = case["select"] if case["kind"] == "selected" else 0
    n_heads = state["q"].shape[1]
    ws = _workspace(state, lambda: cache.workspace_size(seqs.n_seqs, seqs.max_pages, n_heads, select))
    if select:
        cache.attention_selected(seqs, state["q"], state["out"], ws, n_select=select, keep_first=case["first"],
                                 keep_last=case["last"], lse=state["lse"], selected=state["chosen"])
        return {"out": state["out"], "lse": state["lse"], "selected": state["chosen"]}
    cache.attention(seqs, state["q"], state["out"], ws, lse=state["lse"])
    return {"out": state["out"], "lse": state["lse"]}


# ----------------------------------------------------------------------------- plain forms

def _rotate(x, positions, theta):
    """Rotate-half rotary embedding of x [rows, heads, d]; the angles in 64 bits."""
    half = x.shape[-1] // 2
    freq = theta ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    angle = positions.to(torch.float64)[:, None, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)


def _append(state):
    page, theta = state["case"]["page"], state["theta"]
    owner, entry = state["owner"], state["entry"]
    at = state["pages"][owner, entry // page].long()
    slot = entry % page
    new_k = _rotate(state["new_k"], state["positions"], theta)
    state["k"][at, :, slot] = new_k
    state["v"][at, :, slot] = state["new_v"]
    out = {"k": state["k"], "v": state["v"], "q": _rotate(state["q"], state["positions"], theta)}
    if "bounds" in state:
        b, wide = state["bounds"], at[:, None, None].expand(-1, *new_k.shape[1:])
        fresh = at[slot == 0]
        lo, hi = b[:, :, 0].float(), b[:, :, 1].float()
        lo[fresh], hi[fresh] = math.inf, -math.inf
        lo.scatter_reduce_(0, wide, new_k.float(), "amin")
        hi.scatter_reduce_(0, wide, new_k.float(), "amax")
        b.copy_(torch.stack([lo, hi], 2).to(b.dtype))
        out["bounds"] = b
    return out


def _attend(state, see):
    """Attention of q [n, H, d] over the paged entries that ``see`` [n, KV heads, entries] lets through."""
    k, v, q = state["k"], state["v"], state["q"]
    n, H, d = q.shape
    G = k.shape[1]
    pages = state["pages"].clamp(min=0).long()
    keys = k[pages].permute(0, 2, 1, 3, 4).reshape(n, G, -1, d).float()
    s = torch.matmul(q.float().view(n, G, H // G, d), keys.transpose(2, 3).contiguous()) / math.sqrt(d)
    del keys
    s = s.masked_fill(~see[:, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = (s - m).exp()
    total = e.sum(-1, keepdim=True)
    values = v[pages].permute(0, 2, 1, 3, 4).reshape(n, G, -1, d).float()
    out = torch.matmul(e / total, values)
    return out.reshape(n, H, d).to(q.dtype), (m + total.log()).reshape(n, H)


def _seen(state):
    entries = state["pages"].shape[1] * state["case"]["page"]
    at = torch.arange(entries, device=state["pages"].device)
    return (at < state["lengths"][:, None])[:, None].expand(-1, state["k"].shape[1], -1)


def _attention(state):
    out, lse = _attend(state, _seen(state))
    return {"out": out, "lse": lse}


def _selected(state):
    case, q, b = state["case"], state["q"].double(), state["bounds"]
    page, n_select = case["page"], case["select"]
    n, H, d = q.shape
    G, width = b.shape[1], state["pages"].shape[1]
    q = q.view(n, G, H // G, d)
    bounds = b[state["pages"].clamp(min=0).long()].double()        # [n, width, G, 2, d]
    # max(q lo, q hi) of each query head, summed over the heads and channels
    above, below = q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)     # [n, G, d]
    score = ((bounds[:, :, :, 1] * above[:, None]).sum(-1) + (bounds[:, :, :, 0] * below[:, None]).sum(-1)).transpose(1, 2)
    count = ((state["lengths"] + page - 1) // page)[:, None, None]
    at = torch.arange(width, device=q.device)
    score = score.masked_fill((at < case["first"]) | (at >= count - case["last"]), math.inf)
    score = score.masked_fill(at >= count, -math.inf)
    # the n_select best, ties to the lower page: a stable sort by falling score
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :n_select]
    keep = torch.zeros(n, G, width, dtype=torch.bool, device=q.device).scatter_(2, best, True) & (at < count)
    out, lse = _attend(state, _seen(state) & keep.repeat_interleave(page, 2))
    chosen = torch.where(keep, at, width).sort(-1).values
    chosen = torch.nn.functional.pad(chosen, (0, max(0, n_select - width)), value=width)[..., :n_select]
    return {"out": out, "lse": lse, "selected": torch.where(chosen < width, chosen, -1).to(torch.int32)}


def _logprobs(state):
    x, tok, top = state["logits"].float(), state["tokens"].long()[:, None], state["case"]["top"]
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    total = e.sum(-1, keepdim=True)
    lse = m + total.log()
    entropy = (total.log() - (e * (x - m)).sum(-1, keepdim=True) / total)[:, 0]
    mine = x.gather(1, tok)
    ids = torch.arange(x.shape[1], device=x.device)
    rank = 1 + ((x > mine) | ((x == mine) & (ids < tok))).sum(-1)
    # one whole number that orders by value, then by lower id
    bits = (x + 0.0).view(torch.int32).long()
    key = (torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) << 32) | (0x7FFFFFFF - ids)
    best = 0x7FFFFFFF - (key.topk(top, dim=-1).values & 0x7FFFFFFF) if top else tok[:, :0]
    return {"logprob": (mine - lse)[:, 0], "rank": rank.to(torch.int32), "entropy": entropy,
            "top_ids": best.to(torch.int32), "top_logprobs": x.gather(1, best) - lse}


def run(state):
    if own:
        return _framework(state)
    return {"append": _append, "attention": _attention, "selected": _selected, "logprobs": _logprobs}[
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


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "logprobs":
        rows = []
        for i in range(0, case["rows"], 64):
            x, tok = state["logits"][i:i + 64].double(), state["tokens"][i:i + 64].long()
            logp = x - torch.logsumexp(x, 1, keepdim=True)
            mine = logp[torch.arange(len(x), device=x.device), tok]
            order = logp.argsort(dim=1, descending=True, stable=True)[:, :case["top"]]
            rows.append((mine, -(logp.exp() * logp).sum(1), torch.stack([r[o] for r, o in zip(logp, order)])))
        mine, entropy, tops = (torch.cat(c) for c in zip(*rows))
        return {"logprob": mine, "rank": None, "entropy": entropy, "top_ids": None, "top_logprobs": tops}
    page, lens = case["page"], lengths_of(case)
    table = state["pages"].cpu()
    if case["kind"] == "append":
        k, v = state["k"].double(), state["v"].double()
        new_k = _turned(state["new_k"], state["positions"], state["theta"])
        out = {"q": _turned(state["q"], state["positions"], state["theta"])}
        b = state["bounds"].double() if case["bounds"] else None
        row = 0
        for i, length in enumerate(lens):
            m = length if case["chunk"] else 1
            e = length - m
            while e < length:
                p, o = int(table[i, e // page]), e % page
                c = min(page - o, length - e)
                part = new_k[row:row + c].transpose(0, 1)
                k[p, :, o:o + c] = part
                v[p, :, o:o + c] = state["new_v"][row:row + c].double().transpose(0, 1)
                if b is not None:
                    lo, hi = part.amin(1), part.amax(1)
                    b[p, :, 0] = lo if o == 0 else torch.minimum(lo, b[p, :, 0])
                    b[p, :, 1] = hi if o == 0 else torch.maximum(hi, b[p, :, 1])
                e, row = e + c, row + c
        out.update(k=k, v=v)
        if b is not None:
            out["bounds"] = b
        return out
    n, H, d = state["q"].shape
    G = state["k"].shape[1]
    outs, lses = [], []
    for i, length in enumerate(lens):
        count = (length + page - 1) // page
        mine = state["pages"][i, :count].long()
        k = state["k"][mine].double().transpose(0, 1).reshape(G, count * page, d)
        v = state["v"][mine].double().transpose(0, 1).reshape(G, count * page, d)
        q = state["q"][i].double().view(G, H // G, d)
        for h in range(G):
            at = torch.arange(length, device=k.device)
            if case["kind"] == "selected" and count > case["select"]:
                b = state["bounds"][mine, h].double()
                score = torch.maximum(q[h][:, None] * b[:, 0], q[h][:, None] * b[:, 1]).sum((0, 2))
                score[:case["first"]] = math.inf
                score[count - case["last"]:] = math.inf
                kept = score.argsort(descending=True, stable=True)[:case["select"]].sort().values
                at = (kept[:, None] * page + torch.arange(page, device=k.device)).reshape(-1)
                at = at[at < length]
            s = q[h] @ k[h, at].T / math.sqrt(d)
            lse = torch.logsumexp(s, 1)
            outs.append((s - lse[:, None]).exp() @ v[h, at])
            lses.append(lse)
    got = {"out": torch.cat(outs).view(n, H, d), "lse": torch.cat(lses).view(n, H)}
    if case["kind"] == "selected":
        got["selected"] = None
    return got
