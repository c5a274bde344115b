"""Rows of 8-bit codes at the ends of fp32's range."""
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

