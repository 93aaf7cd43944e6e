"""Attention over a paged cache whose Values are infinite, or so large that the sum of a row's Values overflows.

A weight is positive however small, so an infinite Value that a row sees makes its channel that infinity; a weighted mean
is never larger than the largest Value."""
import numpy as np
import pytest

from oracle import paged as OP

from paged_helpers import Case, attention_tolerance, check_attention, f64

pytestmark = pytest.mark.gpu

SHAPES = [  # heads, KV heads, head size, page, dtype
    (4, 4, 64, 16, "bf16"), (8, 2, 128, 16, "bf16"), (20, 1, 64, 32, "bf16"), (4, 2, 32, 16, "f32"),
    (8, 2, 128, 64, "f32"),
]
LENGTHS = [1, 2, 17, 33, 130, 700]      # one part of a row
SPLIT = [5000, 1, 300]                  # several


def attend(case, select):
    out, lse = case.outputs()
    if select:
        case.cache.attention_selected(case.seqs, case.q, out, case.workspace(select), n_select=select, lse=lse)
    else:
        case.cache.attention(case.seqs, case.q, out, case.workspace(), lse=lse)
    return out, lse


def place_infinities(case, seed):
    """Infinite Values in channels of their own: the first entry, the last, one in the middle, and for the KV head's first
    query head the entry of the largest weight.  Returns {(sequence, KV head): {channel: infinity}}."""
    rng = np.random.default_rng(seed)
    q, grp, put = f64(case.q), case.H // case.G, {}
    for i, n in enumerate(case.lens):
        for g in range(case.G):
            k, _ = case.rows(i, g)
            best = int((k @ q[i, g * grp]).argmax())
            channels = rng.permutation(case.d)[:4]
            for ch, e in zip(channels, (0, n - 1, n // 2, best)):
                x = float(rng.choice([-np.inf, np.inf]))
                case.v[int(case.table[i, e // case.page]), g, e % case.page, int(ch)] = x
                put.setdefault((i, g), {})[int(ch)] = x
    return put


def check_infinities(case, out, lse, put):
    """The channels with an infinity are that infinity; every other one, and the log-sum-exp, are what they are."""
    out, lse, q, grp, scale = f64(out), f64(lse), f64(case.q), case.H // case.G, 1.0 / np.sqrt(case.d)
    for (i, g), channels in put.items():
        h = slice(g * grp, (g + 1) * grp)
        k, v = case.rows(i, g)
        for ch, x in channels.items():
            assert (out[i, h, ch] == x).all(), (i, g, ch, x, out[i, h, ch])
        rest = [c for c in range(case.d) if c not in channels]
        o, l, weighted, products = OP.attend(q[i, h], k, v[:, rest], scale)
        tol, ltol = attention_tolerance(case.dtype, len(k), case.d, scale, o, weighted, products)
        assert (np.abs(out[i, h][:, rest] - o) <= tol).all(), (i, g)
        assert (np.abs(lse[i, h] - l) <= ltol + 2.0 ** -22 * np.abs(l)).all(), (i, g)


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("lengths", [LENGTHS, SPLIT], ids=["whole", "split"])
@pytest.mark.parametrize("selected", [False, True], ids=["every page", "chosen pages"])
def test_infinite_values(heads, kv_heads, d, page, dtype, lengths, selected):
    for seed in range(3):
        case = Case(lengths, heads, kv_heads, d, page, dtype, seed=100 * seed + heads, bounds=selected)
        put = place_infinities(case, seed)
        check_infinities(case, *attend(case, case.table.shape[1] if selected else 0), put)


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_a_sequence_of_one_infinite_value(dtype, d):
    """The weight of the only entry is 1."""
    case = Case([1, 1], 4, 2, d, 16, dtype, seed=1)
    case.v[int(case.table[0, 0]), :, 0] = float("inf")
    case.v[int(case.table[1, 0]), :, 0] = -float("inf")
    out, _ = attend(case, 0)
    assert (out[0] == float("inf")).all() and (out[1] == -float("inf")).all()


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("lengths", [LENGTHS, SPLIT], ids=["whole", "split"])
def test_opposite_infinities_are_not_a_number(dtype, d, lengths):
    case = Case(lengths, 4, 2, d, 16, dtype, seed=2)
    for i, n in enumerate(lengths):
        for e, x in ((0, np.inf), (n - 1, -np.inf)):
            case.v[int(case.table[i, e // 16]), :, e % 16, 5] = x
    out, _ = attend(case, 0)
    for i, n in enumerate(lengths):
        assert (out[i, :, 5].isnan() if n > 1 else out[i, :, 5] == -np.inf).all(), n
        assert out[i, :, [c for c in range(d) if c != 5]].isfinite().all()


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("n", [2, 40, 4100])
def test_an_infinite_value_of_a_small_weight(dtype, d, n):
    """A weight of e^-50 of the largest."""
    case = Case([n], 4, 2, d, 16, dtype, seed=3)
    case.q.zero_()
    case.q[:, :, 0] = 10.0
    case.k.mul_(0.0)                         # what no sequence holds stays NaN
    case.k[int(case.table[0, 0]), :, 0, 0] = 5.0
    case.v[int(case.table[0, (n - 1) // 16]), :, (n - 1) % 16, 7] = -float("inf")
    out, lse = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace(), scale=1.0, lse=lse)
    assert (out[0, :, 7] == -float("inf")).all() and out[0, :, 8:].isfinite().all()
    assert (lse == 50.0).all()


@pytest.mark.parametrize("heads, kv_heads, d, page, dtype", SHAPES)
@pytest.mark.parametrize("lengths", [LENGTHS + [0], SPLIT], ids=["whole", "split"])
@pytest.mark.parametrize("selected", [False, True], ids=["every page", "chosen pages"])
def test_values_near_the_largest(heads, kv_heads, d, page, dtype, lengths, selected):
    """Values of one sign and up to 3e38: their sum overflows, their mean does not."""
    import torch
    case = Case(lengths, heads, kv_heads, d, page, dtype, seed=3, bounds=selected)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = 3.0e38 * (0.5 + 0.5 * torch.rand(case.v.shape, generator=g, device="cuda"))
    x[..., 1::2].neg_()
    case.v.copy_(torch.where(case.v.isnan(), case.v, x.to(case.v.dtype)))
    check_attention(case, *attend(case, case.table.shape[1] if selected else 0))


@pytest.mark.parametrize("dtype, d", [("bf16", 64), ("f32", 64)])
def test_small_values(dtype, d):
    """Values down to 1e-30 keep their relative precision."""
    case = Case(LENGTHS + SPLIT, 4, 2, d, 16, dtype, seed=5)
    case.v.mul_(1.0e-30)
    check_attention(case, *attend(case, 0))
