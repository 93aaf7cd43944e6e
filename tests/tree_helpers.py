"""Trees of drafts at the kernel whose waves share tiles: from 256 workgroups of 16 columns on, or under a long table."""
from __future__ import annotations

import contextlib

import paper_2608_08684_amd as rk

from test_gpu_paged_tree import Drafts, make

# (sequences, drafts of the longest tree, query heads to a KV head, columns of a workgroup, table in entries or None)
SHARED = {
    "many-64": (47, 12, 4, 64, None),       # 47 x 2 KV heads x 3 blocks of 16 columns
    "many-128": (24, 12, 8, 128, None),     # 24 x 2 x 6
    "room-64": (3, 16, 4, 64, 1 << 16),     # few short sequences, a table with room for long ones
    "room-128": (2, 20, 12, 128, 1 << 16),  # 240 columns: two workgroups of them
}


def lengths_of(form, longest=200):
    """Sequences from their drafts alone to `longest` entries."""
    n, drafts, *_ = SHARED[form]
    return [longest] + [drafts + (37 * i) % (longest - drafts + 1) for i in range(n - 1)]


def counts_of(form):
    """1 to all drafts; the first tree is the widest."""
    n, drafts, *_ = SHARED[form]
    return [drafts] + [1 + (5 * i) % drafts for i in range(n - 1)]


def shared(form, d, dtype, masks="tree", page=16, seed=0, lengths=None, counts=None, table=None, **kw):
    """A case and its drafts, 2 KV heads."""
    group, entries = SHARED[form][2], table or SHARED[form][4]
    lengths = lengths or lengths_of(form)
    if entries:
        kw["width"] = entries // page
    case = make(lengths, 2 * group, 2, d, page, dtype, seed=seed, **kw)
    return case, Drafts(case, counts or counts_of(form), masks, seed=seed)


@contextlib.contextmanager
def all_shared(calls):
    """Every one of that many attention calls goes to the kernel whose waves share tiles."""
    rk.timing_begin("paged_tree_shared")
    done = False
    try:
        yield
        done = True
    finally:
        launches, _ = rk.timing_end()
    assert not done or launches == calls, f"{launches} of {calls} calls"
