"""8-bit rows under the scale bytes that only a caller writes: Values out of bf16's range, in drafts and in the text."""
import pytest

import paper_2608_08684_amd as rk

from e4m3_helpers import Case8, empty_cache, values
from test_gpu_paged_tree import Drafts, make
from tree_helpers import SHARED, all_shared, shared

pytestmark = pytest.mark.gpu


def beyond(byte):
    """The least code that is infinite as bf16 under a scale byte: code c is 2^(c / 8 - 7) and more, times 2^(byte - 127)."""
    return 8 * (262 - byte)


def of_form(form, d, seed):
    if form == "narrow":
        case = make([70, 90], 8, 2, d, 16, "e4m3", seed=seed)
        return case, Drafts(case, [10, 30], seed=seed)
    case, drafts = shared(form, d, "e4m3", seed=seed)
    with all_shared(1):
        drafts.run()
    return case, drafts


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["narrow", *SHARED])
@pytest.mark.parametrize("byte, sign", [(247, 0), (247, 0x80), (248, 0), (254, 0), (254, 0x80), (246, 0)])
def test_values_beyond_bf16_reach_those_who_see_them(form, d, byte, sign):
    """The rows whose mask leaves the draft out do not change by a bit; the others get the infinity, in its channel
    alone.  The largest code that is finite is no infinity."""
    import torch
    case, drafts = of_form(form, d, seed=11)
    seq, draft, head, channel, other = 0, 2, 1, 7, d - 3
    group = case.H // 2
    u = case.lens[seq] - drafts.counts[seq] + draft
    at = (int(case.table[seq, u // 16]), head, u % 16)
    sees = torch.zeros(len(drafts.q), dtype=torch.bool, device="cuda")
    for j in range(drafts.counts[seq]):
        sees[j] = bool(drafts.words[j] >> draft & 1)
    assert 0 < int(sees.sum()) < drafts.counts[seq]
    mine = torch.zeros(case.H, dtype=torch.bool, device="cuda")
    mine[head * group:(head + 1) * group] = True
    hit = sees[:, None] & mine
    codes = case.raw["v"].view(torch.uint8)
    codes[at] = 0
    case.raw["v_scales"][at] = byte
    ref, ref_lse = drafts.run()
    assert ref.isfinite().all()
    code = beyond(byte) if byte > 246 else 0x7E
    codes[at][channel] = code | sign
    codes[at][other] = (code - 1) | sign             # the largest that is finite: 1.875 2^127, or less
    out, lse = drafts.run()
    assert torch.equal(out[~hit], ref[~hit]) and torch.equal(lse, ref_lse)
    got = out[hit]
    if byte > 246:
        assert (got[:, channel] == (-float("inf") if sign else float("inf"))).all()
    assert got[:, other].isfinite().all() and (got[:, other] < 0 if sign else got[:, other] > 0).all()
    rest = [x for x in range(d) if x not in (channel, other)]
    assert torch.equal(got[:, rest], ref[hit][:, rest])


@pytest.mark.parametrize("form", ["narrow", *SHARED])
def test_both_infinities_and_nan(form):
    """A draft with both infinities beside finite values and NaN, each in a channel of its own."""
    import torch
    case, drafts = of_form(form, 64, seed=12)
    draft = 3
    u = case.lens[0] - drafts.counts[0] + draft
    at = (int(case.table[0, u // 16]), 0, u % 16)
    codes = case.raw["v"].view(torch.uint8)
    codes[at] = 0
    case.raw["v_scales"][at] = 250
    for channel, code in ((1, 0x60), (2, 0xE0), (3, 0x7F), (4, 0x7E), (5, 0xFE), (6, 0x5F), (7, 0xDF)):
        codes[at][channel] = code
    out, _ = drafts.run()
    group, inf = case.H // 2, float("inf")
    for j in range(drafts.counts[0]):
        got = out[j, :group].float()
        if drafts.words[j] >> draft & 1:
            assert (got[:, 1] == inf).all() and (got[:, 2] == -inf).all() and got[:, 3].isnan().all()
            assert (got[:, 4] == inf).all() and (got[:, 5] == -inf).all() and got[:, [0, *range(6, 64)]].isfinite().all()
        else:
            assert got.isfinite().all()
    assert out[drafts.counts[0]:].isfinite().all() and out[:, group:].isfinite().all()


@pytest.mark.parametrize("d", [64, 128])
def test_every_code_under_every_scale_byte(d):
    """Bytes 1 .. 254: read back as the nearest bf16 numbers, and infinities from 2^128 on."""
    import torch
    page, per = 256, 256 // d
    cache = empty_cache(per, 1, page, d)
    cache.k.view(torch.uint8).copy_(torch.arange(256, dtype=torch.uint8, device="cuda").view(per, 1, 1, d))
    cache.v.view(torch.uint8).copy_(cache.k.view(torch.uint8).flip(-1))
    cache.k_scales.copy_(torch.arange(page, device="cuda").clamp(1, 254).to(torch.uint8))
    cache.v_scales.copy_(cache.k_scales.flip(-1))
    seqs = rk.PagedSeqs(torch.arange(per, dtype=torch.int32, device="cuda")[None],
                        torch.tensor([per * page], dtype=torch.int32, device="cuda"))
    k = torch.empty(per * page, 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache.read(seqs, k, v, row_offsets=[0, per * page])
    for got, held, scales in ((k, cache.k, cache.k_scales), (v, cache.v, cache.v_scales)):
        want = values(held, scales).view(-1, d).cpu().bfloat16()    # 4 bits of the value: one rounding at most
        got = got[:, 0].cpu()
        assert ((got == want) | (got.isnan() & want.isnan())).all() and got.isinf().any()


@pytest.mark.parametrize("length", [40, 3000])
def test_infinite_values_of_the_text(length):
    """One new token over Values beyond bf16's range: those infinities, in their channels alone."""
    import torch
    case = Case8([length, 33], 8, 2, 64, 16, seed=13)
    codes = case.raw["v"].view(torch.uint8)
    at = (int(case.table[0, 1]), 1, 3)
    codes[at], case.raw["v_scales"][at] = 0, 251
    ref, _ = case.outputs()
    case.cache.attention(case.seqs, case.q, ref, case.workspace())
    codes[at][5], codes[at][6], codes[at][7] = 0x58, 0xFE, 0x57       # 2^128, below -2^128, 1.875 2^127
    out, _ = case.outputs()
    case.cache.attention(case.seqs, case.q, out, case.workspace())
    got = out[0, 4:]
    assert (got[:, 5] == float("inf")).all() and (got[:, 6] == -float("inf")).all() and got[:, 7].isfinite().all()
    rest = [x for x in range(64) if x not in (5, 6, 7)]
    assert (got[:, rest] == ref[0, 4:][:, rest]).all() and (out[0, :4] == ref[0, :4]).all() and (out[1] == ref[1]).all()
