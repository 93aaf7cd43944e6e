"""Token log probabilities of many long rows: workgroups of 256 and 512 threads over several passes of a row, against
float64."""
import numpy as np
import pytest

from oracle import paged as OP

from paged_helpers import f64
from test_gpu_token_logprobs import logits, run

pytestmark = pytest.mark.gpu

CALLS = [(600, 20011, 3), (300, 50257, 1)]     # 256 threads a row, 512: rows, vocabulary, padding


def check_row(x, token, n_top, out, r, bf16, independent=False):
    """How far a row's results may be off.  With d = x - max, p the probabilities, S and T as in the kernel, m = |T| / S:

    S and T are off by `sums` of themselves: every addition rounds by 2^-24, and a term goes through those of a pass (16 or
    32), of the thread's passes and 6 for the lanes, 6 for the waves and 6 for the parts of a row.  Where the logits are noise
    the roundings are too: at least 256 chains of either sign average out and the last joins are left, two steps.
    A weight e^d other than the largest is off by |d| (2^-24 for the difference, 2^-24 for its product with log2(e), 2^-26 for
    log2(e) in 24 bits) and 2^-23 for the exponential, together under (|d| + 1) 2^-22; it moves log S by p times that and the
    entropy by p (1 + |d| + m) times that.  In noise, 2^-26 is left: m of it, and the differences' variance.
    log S, T / S and the result are rounded: 2^-23 of each."""
    lp, rank, h, ids, top = OP.logprobs(x, token, n_top)
    seen = x > -np.inf
    with np.errstate(invalid="ignore"):
        d = x[seen] - x[ids[0] if n_top else x.argmax()]
    p = np.exp(d)
    log_s, p = np.log(p.sum()), p / p.sum()
    m, square, rest = abs((p * d).sum()), (p * d * d).sum(), 1.0 - p[d == 0].sum()
    per_pass = 32 if bf16 else 16
    if independent:
        sums, weights, moved = 2.0 ** -22, 2.0 ** -26 * m, 2.0 ** -26 * (square - m * m)
    else:
        sums = (per_pass + len(x) / (256 * per_pass) + 1 + 18) * 2.0 ** -24
        weights, moved = 2.0 ** -22 * (m + rest), 2.0 ** -22 * (m + square + m * m + rest * (1 + 2 * m))
    step = 2.0 ** -23
    tol = sums + weights + step * log_s
    got = {k: v[r].cpu().numpy() for k, v in out.items()}
    assert got["rank"] == rank, r
    if np.isfinite(lp):
        assert abs(got["logprob"] - lp) <= tol + step * abs(lp), (r, got["logprob"], lp)
    else:
        assert got["logprob"] == lp, r
    bound = sums * (1 + 2 * m) + moved + step * (log_s + m + h)
    assert abs(got["entropy"] - h) <= bound, (r, got["entropy"], h, bound)
    if n_top:
        assert got["top_ids"].tolist() == ids, r
        for a, b in zip(got["top_logprobs"], top):
            assert a == b if b == -np.inf else abs(a - b) <= tol + step * abs(b), (r, a, b)


def special_rows(x, tok):
    """Rows in which equal or many large logits make the choice of the best harder than group maxima settle it."""
    import torch
    rows, vocab = x.shape
    g = torch.Generator(device="cuda").manual_seed(1)
    ramp = torch.arange(vocab, device="cuda")
    x[1] = 1.5                                                   # every logit the same
    x[2] = torch.randint(-2, 3, (vocab,), generator=g, device="cuda").to(x.dtype)
    x[3] = (-(ramp // 64)).to(x.dtype)                           # falling, rising, in runs
    x[4] = (ramp // 64).to(x.dtype)
    x[5] = -float("inf")                                         # fewer that count than are asked for
    x[5, [7, vocab // 2, vocab - 1]] = torch.tensor([1.0, 1.0, 0.5], device="cuda", dtype=x.dtype)
    x[6, vocab // 3:2 * vocab // 3] = 25.0                       # more large logits than a list holds
    x[6, vocab // 2] = 26.0
    x[7, :vocab - 5] = torch.finfo(x.dtype).min                  # a mask of the type's lowest value
    x[8, :vocab - 40] = -float("inf")
    x[9, -33:] = 30.0                                            # one more than the most that is asked for
    x[10, ::vocab // 31] = 30.0                                  # one in every so many, far apart
    for r, t in ((1, vocab - 1), (2, vocab // 2), (3, 64), (4, vocab - 3), (5, vocab // 2), (6, 2 * vocab // 3 - 1),
                 (7, 0), (8, vocab - 1), (9, vocab - 33), (10, 0)):
        tok[r] = t
    return list(range(12))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, pad", CALLS)
@pytest.mark.parametrize("n_top", [0, 5, 32])
def test_many_long_rows(dtype, rows, vocab, pad, n_top):
    x, tok = logits(rows, vocab, dtype, n_top + 1, pad=pad, shift=1)
    look = special_rows(x, tok) + [rows // 2, rows - 2, rows - 1]
    out = run(x, tok, n_top)
    for r in look:
        check_row(f64(x[r]), int(tok[r]), n_top, out, r, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, pad", CALLS + [(3, 128256, 0)])
def test_confident_rows_keep_their_digits(dtype, rows, vocab, pad):
    """One logit 8 to 40 above the others, anywhere in its row."""
    import torch
    x, tok = logits(rows, vocab, dtype, 3, pad=pad)
    x.zero_()
    for r in range(rows):
        tok[r] = (r * 7919 + 4321) % vocab
        x[r, int(tok[r])] = 8.0 + 0.5 * (r % 65)
    out = run(x, tok, 2)
    for r in range(0, rows, max(1, rows // 67)):
        check_row(f64(x[r]), int(tok[r]), 2, out, r, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(600, 20011), (300, 50257), (1024, 128256), (16, 128256), (1, 1 << 22)])
def test_sums_of_a_language_model_s_logits(dtype, rows, vocab):
    """A bulk and a few likely tokens far above it."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, vocab, generator=g, device="cuda").mul_(2.0)
    likely = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
    x.scatter_add_(1, likely, torch.rand(rows, 24, generator=g, device="cuda") * 12.0)
    x, tok = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32), likely[:, 3].to(torch.int32)
    out = run(x, tok, 20)
    for r in sorted({0, rows // 3, rows - 1}):
        check_row(f64(x[r]), int(tok[r]), 20, out, r, dtype == "bf16", independent=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, threads", [(600, 256), (300, 512), (40, 1024)])
def test_two_logits_of_one_thread(dtype, rows, threads):
    """All others have no probability: S = 1 + e^-D takes one rounding, T = -D e^-D is small, and with log S the results are
    off by two steps at most, however far the second logit of the thread lies above the first (up to 44)."""
    import torch
    apart = threads * (8 if dtype == "bf16" else 4)      # the thread's vectors of a pass and of the next
    x = torch.full((rows, 9 * apart + 5), -float("inf"), device="cuda")
    lead = 8.0 + 0.125 * (torch.arange(rows) % 289)
    at = apart * (1 + torch.arange(rows) % 8) + 1
    x[:, 1] = 0.0
    x[torch.arange(rows), at] = lead.cuda()
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    out = run(x, at.to(torch.int32).cuda(), 0)
    e = np.exp(-lead.double().numpy())
    assert (np.abs(f64(out["logprob"]) + np.log1p(e)) <= 2.0 ** -22).all()
    h = np.log1p(e) + lead.numpy() * e / (1 + e)
    assert (np.abs(f64(out["entropy"]) - h) <= 2.0 ** -22 + 2.0 ** -23 * h).all(), np.abs(f64(out["entropy"]) - h).max()
