"""Attention over the paged cache where numbers are extreme: against float64
(oracle/paged_oracle.py), or against what the formula gives exactly."""
import pytest
import torch

from test_gpu_paged import BF, HF, NAN, attend, check, make, queries

pytestmark = pytest.mark.gpu


def rows_at(cache, length, s=0):
    """Page and row of a sequence's first slots, to index the pools by."""
    slot = torch.arange(length, device="cuda")
    page = cache.page_size
    return cache.table[s].long()[slot // page], slot % page


@pytest.mark.parametrize("rows, length", [(1, 100), (1, 40000), (90, 40000), (200, 300), (200, 40000)])
def test_weights_that_vanish_carry_what_is_not_finite(rows, length):
    """Half of the slots 181 nats below the others, one of them with a NaN or an infinity
    in V: it reaches the output (0 times it is NaN), whether a unit is one piece or several
    that are joined."""
    cache = make([length], 2, 64)
    at = rows_at(cache, length)
    sign = torch.where(torch.arange(length, device="cuda") < length // 2, -1.0, 1.0)
    cache.k_pages[at] = sign[:, None, None].to(BF).expand(length, 2, 128)
    q = torch.full((rows, 8, 128), 8.0, dtype=BF, device="cuda")
    clean, clean_lse, _ = attend(cache, q)
    assert torch.isfinite(clean).all()
    slot = min(20, length - rows)  # seen by every token
    page, row = at[0][slot], at[1][slot]
    for value in (NAN, float("inf")):
        cache.v_pages[page, row, 1, 77] = value
        out, lse, _ = attend(cache, q)
        assert not torch.isfinite(out[:, 4:, 77]).any()  # (an infinity where a token sees no other slots)
        out[:, 4:, 77] = clean[:, 4:, 77]
        assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("rows, length", [(1, 5), (1, 40000), (90, 200), (200, 300), (200, 40000)])
def test_logits_of_minus_infinity(rows, length):
    """A token all of whose slots have a logit of -infinity has a sum of 0: its output is
    NaN (0 / 0) and its log-sum-exp -infinity; tokens with another slot are not touched."""
    cache = make([length], 2, 64)
    at = rows_at(cache, length)
    cache.k_pages[at[0], at[1], 1, 3] = -float("inf")
    q = queries(rows, 8, BF).abs() + 0.25  # (no 0 times infinity)
    out, lse, _ = attend(cache, q)
    assert torch.isfinite(out[:, :4]).all() and torch.isfinite(lse[:4]).all()
    assert torch.isnan(out[:, 4:]).all() and (lse[4:] == -float("inf")).all()
    # the last slot, which the last token alone sees, as any other
    cache.k_pages[at[0][-1], at[1][-1], 1, 3] = 1.0
    out, lse, _ = attend(cache, q)
    last = cache.v_pages[at[0][-1], at[1][-1], 1]
    assert torch.equal(out[-1, 4:], last.expand(4, 128)) and torch.isfinite(lse[4:, -1]).all()
    assert torch.isnan(out[:-1, 4:]).all() and (lse[4:, :-1] == -float("inf")).all()


@pytest.mark.parametrize("dtype, size, scale", [(BF, 1.0, 2.0 ** 40), (BF, 1.0, 2.0 ** 96), (BF, 60000.0, 128 ** -0.5),
                                                (HF, 1.0, 2.0 ** 30), (HF, 1.0, 2.0 ** 96),
                                                (HF, 3000.0, 128 ** -0.5), (HF, 60000.0, 128 ** -0.5)])
@pytest.mark.parametrize("rows, length", [(1, 300), (1, 9000), (200, 300), (200, 9000)])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_far_from_zero(dtype, size, scale, rows, length, sign):
    """Where fp32's steps of a logit are more than 1 the slots with the largest one have
    all the weight: one slot's V, bit by bit, or the average of two equal ones."""
    cache = make([length], 1, 64, dtype)
    at = rows_at(cache, length)
    best, other = length // 3 if length > 2 * rows else 20, 7
    k = cache.k_pages[at]
    k[:] = 0.5 * size if sign > 0 else size
    k[best] = size if sign > 0 else 0.5 * size
    cache.k_pages[at] = k
    gen = torch.Generator().manual_seed(0)
    q = ((torch.rand((rows, 4, 128), generator=gen) * 0.5 + 0.5) * size * sign).to(dtype).cuda()
    v = cache.v_pages[at][:, 0]
    out, lse, status = attend(cache, q, scale=scale)
    assert status == 0 and torch.equal(out, v[best].expand(rows, 4, 128))
    want = (q.double() @ k[best, 0].double() * scale).T
    # (2^-20 of the terms' magnitudes for the logit, all of one sign here; 2^-22 for the rest)
    assert ((lse.double() - want).abs() <= (2.0 ** -20 + 2.0 ** -22) * want.abs()).all()
    k[other] = k[best]
    cache.k_pages[at] = k
    out, _, _ = attend(cache, q, scale=scale)
    both = (v[best].double() + v[other].double()) / 2
    half = torch.finfo(dtype).eps / 2
    # a half each, exactly; sums of two in fp32, and the output's rounding
    assert ((out.double() - both).abs() <= (half + 2.0 ** -22) * both.abs() + 2.0 ** -22 * v[best].double().abs()).all()


@pytest.mark.parametrize("rows, logit, sd", [(1, 18.0, 0.0), (1, 16.0, 1.0), (3, 17.0, 0.5), (130, 18.0, 0.0),
                                             (130, 16.0, 1.0)])
def test_f16_keeps_the_tail_behind_a_sink(rows, logit, sd):
    """A sink with 99 % of the mass or more and V = 0: the output is what tens of thousands
    of slots with probabilities about 2^-25 of the largest add up to.  (As many heads as a
    cache has, so that pieces are long: each has a reference of its own.)"""
    length, h = 32768, 64
    cache = make([length], h, 256, HF)
    at = rows_at(cache, length)
    gen = torch.Generator().manual_seed(1)
    u = torch.randn(128, generator=gen)
    one = u * 128 ** 0.5 / u.dot(u)  # a logit of 1
    k = torch.randn((length, 1), generator=gen) * sd * one
    k[0] = one * logit
    cache.k_pages[at] = k.to(HF).cuda()[:, None]
    v = torch.rand((length, 128), generator=gen) + 0.5
    v[0] = 0.0
    cache.v_pages[at] = v.to(HF).cuda()[:, None]
    q = u.to(HF).cuda().expand(rows, h, 128).contiguous()
    out, lse, _ = attend(cache, q)
    check(cache, q, out, lse, [0, rows])
