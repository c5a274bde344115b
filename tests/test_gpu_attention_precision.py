"""Attention over a paged cache at the ends of its numbers: probabilities held to 24 bits whatever the results' type, values up to the largest ones."""
import math

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import BF16, E4M3, FP32, ULP, Paged, assert_near, attended, gen, half_step, values

pytestmark = pytest.mark.gpu


def _split(x):
    """The nearest bf16 values of fp64 numbers, and of what they leave."""
    a = x.to(BF16).double()
    return a, (x - a).to(BF16).double()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_probabilities_are_not_rounded_to_16_bits(cache, dtype):
    """Three positions with the weights 1, e^s and 1 and the values -a, 1 and -b, a + b being e^s to two bf16 terms: what is left over, more than 2^-19 of e^s in all of
    these cases, is the result, and nothing is left where the weights have two terms themselves.

    Half steps of fp32 that e^s may be off, relative: 2 |s| of its exponent (the factor to units of log 2, the product; all other products are of powers of 2 and one number),
    2 of the exponential, 1 of the scale of an 8-bit row.  The products are exact; the first terms' sum has four addends of at most e^s that the matrix instruction may cut off by a
    step each, 8, those of the smaller terms 2^-8 of that: 9.  The quotient and its divisor 4 of the result."""
    s = -torch.linspace(0.25, 1.0, 3001, dtype=torch.float64).to(BF16).double().unique()
    e = torch.exp(s)
    a, b = _split(e)
    s = s[((e - a - b).abs() > 2.0 ** -19 * e)]
    e = torch.exp(s)
    a, b = _split(e)
    n = s.numel()
    assert n >= 20
    p = Paged([3] * n, 4, 1, 16, cache, seed=1)
    score = torch.stack([torch.zeros(n), s.float(), torch.zeros(n)], dim=1)
    value = torch.stack([-a.float(), torch.ones(n), -b.float()], dim=1)
    for i in range(n):
        page, off = p.slots(i, torch.arange(3))
        page, off = page.cuda(), off.cuda()
        for t, scale, x in ((p.k, p.k_scale, score[i]), (p.v, p.v_scale, value[i])):
            # of 8 bits: the code of 1 or -1, and the number's magnitude as the scale
            entry = x if cache is BF16 else torch.where(x < 0, -1.0, 1.0)
            rows = entry[:, None, None].repeat(1, 1, 16)
            if t is p.k:
                rows[:, :, 1:] = 0.0
            if cache is BF16:
                t[page, :, off] = rows.to(BF16).cuda()
            else:
                t.view(torch.uint8)[page, :, off] = rows.to(E4M3).view(torch.uint8).cuda()
                scale[page, :, off] = x.abs()[:, None].cuda()
    q = torch.zeros((n, 2, 16))
    q[:, :, 0] = 1.0
    out = mm.DecodeAttention(p.cache, 2, scale=1.0)(q.to(dtype).cuda(), p.table.cuda(), torch.full((n,), 3, dtype=torch.int32, device="cuda"), 3).cpu().double()
    want = ((e - a - b) / (2.0 + e))[:, None, None]
    bound = (e * (2 * s.abs() + 2 + 1 + 9) * ULP / (2.0 + e))[:, None, None] + want.abs() * (4 * ULP + half_step(dtype))
    assert ((out - want).abs() <= bound).all(), float(((out - want).abs() / bound).max())


@pytest.mark.parametrize("lengths, max_len", [([1, 2, 40, 700], 700), ([1, 33, 5000, 3000], 5000), ([60] * 70 + [1, 2, 33], 64), ([9000], 40000)])
@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP32, BF16), (FP32, FP32), (BF16, E4M3), (FP32, E4M3)])
@pytest.mark.parametrize("size", [3e38, 2.0 ** -100])
def test_values_of_any_size_have_a_mean(lengths, max_len, dtype, cache, size):
    """A weighted mean is no larger than its largest value, however many there are, whatever the order of the scores, in one part and in several."""
    p = Paged(lengths, 16, 2, 64, cache, seed=1)
    kv = p.fill(2, k_gain=3.0)
    for s, n in enumerate(lengths):
        page, off = (t.cuda() for t in p.slots(s, torch.arange(n)))
        order = kv[s][0][:, :, 0].sum(dim=1).argsort(descending=s % 2 == 1)      # scores that rise or fall with the first channel
        at = page[order.cuda()], off[order.cuda()]
        p.k.view(torch.uint8)[page, :, off] = p.k.view(torch.uint8)[at[0], :, at[1]]
        if cache is E4M3:
            p.k_scale[page, :, off] = p.k_scale[at[0], :, at[1]]
        k = kv[s][0][order]
        x = (0.9 + 0.1 * torch.rand((n, 2, 64), generator=gen(3 + s))) * size
        x[:, :, 32:] *= torch.where(torch.rand((n, 2, 32), generator=gen(4 + s)) < 0.5, -1.0, 1.0)
        if cache is E4M3:
            codes, sc = (x / x.abs().amax(dim=-1, keepdim=True) * 448).to(E4M3), (x.double().abs().amax(dim=-1) / 448).float()
            p.v.view(torch.uint8)[page, :, off], p.v_scale[page, :, off] = codes.view(torch.uint8).cuda(), sc.cuda()
            v = values(codes, sc)
        else:
            p.v[page, :, off] = x.to(cache).cuda()
            v = values(x.to(cache))
        kv[s] = k, v
    q = torch.randn((len(lengths), 6, 64), generator=gen(5)).to(dtype)
    q[:, :, 0] += 2.0
    q = q.to(dtype)
    lse = torch.zeros((len(lengths), 6), device="cuda")
    out = mm.DecodeAttention(p.cache, 6)(q.cuda(), p.table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max_len, lse=lse)
    assert torch.isfinite(out).all()
    for s in range(len(lengths)):
        want, want_lse, err, lse_err = attended(q[s], kv[s], 0.125)
        assert_near(out[s], want, err, dtype)
        assert ((lse[s].cpu().double() - want_lse).abs() <= lse_err).all()
