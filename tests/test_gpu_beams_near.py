"""Beams whose best candidates lie nearer to each other than fp32 sums can tell."""
import math

import numpy as np
import pytest

from oracle import paged as OP

from paged_helpers import f64
from test_gpu_beams import logits, run

pytestmark = pytest.mark.gpu


def log_sum_bound(x):
    """How far a row's log S may be off.  Sums and logarithm are in doubles (1e-13 for what they round).  A logit below
    the row's largest, M, counts by an exponential and by the factors that move it up to M.  Their arguments, M - x
    together, are rounded as differences and as products, 2^-24 of them each; each exponential is good to an ulp or
    two, 2^-22, and there are one for each time that the thread's largest logit has moved (once a pass of 4096
    logits at the most) and four more.  The largest logits' own exponentials and factors are 1."""
    x = x[x > -np.inf]
    d = x.max() - x
    p = np.exp(-d)
    p, d = p[d > 0] / p.sum(), d[d > 0]
    return float((p * d).sum()) * 2.0 ** -23 + float(p.sum()) * (len(x) / 4096 + 5) * 2.0 ** -22 + 1e-13


def exact_best(x):
    m = x.max()
    return -math.log(math.fsum(np.exp(x - m)))      # the largest logit's log probability


def near_score(rows, first, rng):
    """(score of the second beam, gap): within a few fp32 steps of a tie of the rows' best tokens, on either side, and
    the gap, of the first beam over the second, beyond what their log sums may be off."""
    slack = sum(log_sum_bound(x) for x in rows) + 1e-13
    tie = first + exact_best(rows[0]) - exact_best(rows[1])
    score = np.float32(tie)
    for _ in range(int(rng.integers(0, 2))):
        score = np.nextafter(score, np.float32(9))
    while abs(tie - float(score)) <= slack:
        score = np.nextafter(score, np.float32(-9))
    return float(score), tie - float(score)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups, vocab", [(64, 5000), (100, 333), (40, 50257), (6, 128256), (1, 128256), (1, 600011)])
def test_pairs_of_beams(groups, vocab, dtype):
    """Rows of one likely token each, as a language model sure of itself leaves them: their log sums are good to some
    1e-10, where a float next to 1 is not."""
    import torch
    rng = np.random.default_rng(vocab)
    x = logits(2 * groups, vocab, dtype, vocab, pad=3, shift=1)
    x.clamp_(-9, 9)
    likely = torch.from_numpy(rng.integers(0, vocab, (2 * groups, 1))).cuda()
    x.scatter_(1, likely, torch.from_numpy(rng.uniform(24, 28, (2 * groups, 1))).cuda().to(x.dtype))
    rows, scores, sides = f64(x), np.zeros((groups, 2)), []
    for i in range(groups):
        scores[i, 0] = np.float32(-5 * rng.random())
        scores[i, 1], gap = near_score(rows[2 * i:2 * i + 2], scores[i, 0], rng)
        assert abs(gap) < 2e-6
        sides.append(gap > 0)
    s = torch.from_numpy(scores).float().cuda()
    parents, tokens, best = (t.cpu().numpy() for t in run(x, s, 2))
    for i in range(groups):
        want = OP.beam_select(rows[2 * i:2 * i + 2], scores[i], None, -1, 2)
        assert [(int(a), int(b)) for a, b in zip(parents[i], tokens[i])] == [w[:2] for w in want], (i, sides[i])
    assert groups == 1 or 0 < sum(sides) < groups


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups, beams, vocab, n_out", [
    (3, 4, 1000, 8), (1, 4, 50257, 4), (16, 8, 20000, 16), (1, 1, 128256, 32), (1, 2, 1100003, 8), (300, 2, 500, 2),
    (2, 32, 999, 32), (1, 5, 1, 3),
])
def test_order_and_scores(groups, beams, vocab, n_out, dtype):
    """Parents and tokens as in float64, and its scores but for a log sum's bound and one rounding."""
    import torch
    x = logits(groups * beams, vocab, dtype, vocab + beams)
    s = (-5.0 * torch.rand(groups, beams, generator=torch.Generator().manual_seed(beams))).cuda()
    parents, tokens, best = (t.cpu().numpy() for t in run(x, s, n_out))
    rows, sc = f64(x), f64(s)
    for i in range(groups):
        mine = rows[i * beams:(i + 1) * beams]
        want, bound = OP.beam_select(mine, sc[i], None, -1, n_out), [log_sum_bound(r) for r in mine]
        for a, b in zip(want, want[1:]):        # the inputs leave no doubt
            assert a[0] == b[0] or b[2] == -math.inf or a[2] - b[2] > bound[a[0]] + bound[b[0]]
        assert [(int(a), int(b)) for a, b in zip(parents[i], tokens[i])] == [w[:2] for w in want]
        for j, w in enumerate(want):
            assert best[i, j] == w[2] or abs(best[i, j] - w[2]) <= 2.0 ** -24 * abs(w[2]) + bound[w[0]]


def test_extreme_logits():
    """Masks of the type's lowest value and of -inf, one token alone, equal rows, logits of 1e30."""
    import torch
    x = torch.randn(2 * 6, 700, generator=torch.Generator().manual_seed(6)) * 3
    x[0, 1:] = torch.finfo(torch.float32).min
    x[1, 1:] = -float("inf")
    x[2] = -float("inf")
    x[2, 9] = -3.0
    x[3] = torch.finfo(torch.float32).min
    x[4] = x[5] = 0.0
    x[6], x[7, 3] = 1e30, 1e30
    x[8], x[9] = -1e30, 1e-30
    x[10], x[11, 5] = -float("inf"), float("nan")
    x = x.cuda()
    s = torch.tensor([[-1.0, -1.0 - 2 ** -23], [0.0, -5.0], [-1.0, -1.0], [0.0, -2.0], [-1.0, 0.5], [0.0, 0.0]]).cuda()
    parents, tokens, best = (t.cpu().numpy() for t in run(x, s, 4))
    rows, sc = f64(x), f64(s)
    for i in range(6):
        want = OP.beam_select(rows[2 * i:2 * i + 2], sc[i], None, -1, 4)
        assert [(int(a), int(b)) for a, b in zip(parents[i], tokens[i])] == [w[:2] for w in want], i
        for j, w in enumerate(want):
            assert best[i, j] == np.float32(w[2]) or abs(best[i, j] - w[2]) <= 2.0 ** -24 * abs(w[2]) + 1e-13
