"""Rows of 8-bit codes at the ends of fp32's range and beside the borders between two codes."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import E4M3, ULP, gen

pytestmark = pytest.mark.gpu
FLT_MAX = float(torch.finfo(torch.float32).max)


def _stored(rows):
    """rows [positions, channels] fp32 stored as keys and as values -> their codes (as E4M3 values) and scales, both twice."""
    n, dim = rows.shape
    page = max(4, 1 << (n - 1).bit_length())
    cache = mm.KvCache.empty(1, page, 1, dim, dtype=E4M3)
    x = rows[:, None, :].cuda()
    cache.append(x, x.clone(), torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros((1, 1), dtype=torch.int32, device="cuda"),
                 seq=torch.zeros(n, dtype=torch.int32, device="cuda"))
    return [(t.view(torch.uint8).cpu()[0, 0, :n].view(E4M3).float(), s.cpu()[0, 0, :n]) for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]


@pytest.mark.parametrize("dim", [16, 48, 64, 128, 256])
def test_rows_of_every_size(dim):
    """Finite rows have finite codes whose largest one is 448, up to the largest number and down to those with few bits.

    Of the exact quotient: half a step of e4m3 (2^-4, of its smallest codes 2^-10) and half a step of fp32 of its rounding, of which the last step's own error is far below another
    half; scales are one quotient, of denormal ones 2^-150."""
    sizes = [FLT_MAX, 3e38, 2.0 ** 127, 1e38, 7.7e35, 7.5e35, 1e33, 1.1e30, 1e30, 9e29, 1.0, 1e-20, 1.1e-30, 1e-30, 9e-31, 1e-36, 2.0 ** -126, 1e-38, 1e-40, 1e-43]
    rows = (torch.rand((len(sizes), dim), generator=gen(dim)) * 2 - 1).double() * torch.tensor(sizes, dtype=torch.float64)[:, None]
    rows[:, 3], rows[:, 5], rows[:, 7] = torch.tensor(sizes), 0.0, -torch.tensor(sizes)
    rows = rows.float()
    for codes, scale in _stored(rows):
        most = rows.double().abs().amax(dim=1)
        assert ((scale.double() - most / 448).abs() <= most / 448 * ULP + 2.0 ** -150).all()
        assert torch.isfinite(codes).all() and (codes[:, 3] == 448).all() and (codes[:, 7] == -448).all() and (codes[:, 5] == 0).all()
        exact = rows.double() * 448 / most[:, None]
        assert ((codes.double() - exact).abs() <= torch.clamp(exact.abs() * 2.0 ** -4, min=2.0 ** -10) + exact.abs() * 2 * ULP).all()


def test_codes_beside_their_borders():
    """The nearest code of the nearest fp32 quotient, for numbers that lie as close to the middle between two codes as fp32 has them.  Quotients within 2^-10 steps of the middle
    between two fp32 numbers are left out: the kernel rounds a sum whose second addend is 2^-24 of itself off."""
    codes = sorted({float(c) for c in torch.arange(0x7f, dtype=torch.uint8).view(E4M3).float()})
    middles = np.array([(a + b) / 2 for a, b in zip(codes, codes[1:])])
    rng = np.random.default_rng(1)
    largest = (rng.uniform(1.0, 2.0, 40) * 2.0 ** rng.integers(-20, 20, 40)).astype(np.float32)
    rows, want, sure = [], [], []
    for m in largest:
        near = (middles * float(m) / 448).astype(np.float32)
        for step in (-2, -1, 0, 1, 2):
            y = near.copy()
            for _ in range(abs(step)):
                y = np.nextafter(y, np.float32(math.copysign(1e30, step)))
            y = np.minimum(y, m)
            row, exact = np.zeros(128, np.float32), [Fraction(float(v)) * 448 / Fraction(float(m)) for v in y]
            row[:126], row[127] = y, m
            q = np.array([np.float32(float(e)) for e in exact])      # to 53 bits, then to 24: the same unless beside a middle, see below
            ok = np.ones(128, bool)
            for i, (e, f) in enumerate(zip(exact, q)):
                other = np.nextafter(f, np.float32(1e30 if Fraction(float(f)) < e else 0))
                gap = abs(Fraction(float(other)) - Fraction(float(f)))
                ok[i] = abs(abs(e - Fraction(float(f))) - gap / 2) > gap / 1024
            w = np.zeros(128, np.float32)
            w[:126], w[127] = torch.from_numpy(q).to(E4M3).float().numpy(), 448.0
            rows.append(row), want.append(w), sure.append(ok)
    rows, want, sure = (torch.from_numpy(np.stack(t)) for t in (rows, want, sure))
    assert sure.float().mean() > 0.9
    for got, _ in _stored(rows):
        wrong = (got != want) & sure
        assert not wrong.any(), (int(wrong.sum()), rows[wrong.any(1)][:1], got[wrong][:5], want[wrong][:5])
