"""Log probabilities of rows whose largest entries are many and come late: a wave's reference then lies below them."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from test_gpu_output_head import BF16, FP32, _reference, _tokens

pytestmark = pytest.mark.gpu
LEAD = 20.0                                                  # how far above a wave's reference entries may lie


def _wider(z, tokens, n, lead):
    """The definition's values with bounds for references up to `lead` below the largest entry m.

    u = 2^-24.  Every entry but one may then be a term e^(z - ref) instead of e^(z - m): its exponent is larger by up to `lead`, which costs 3 u
    `lead` (difference, product with log2 e of two roundings), and the sum is multiplied by e^(ref - m) in up to two steps, 3 u `lead` and 2 x (2 + 1) u
    for exponentials and products.  Equal largest entries are such terms too, with the 2 u and the links of the others, so of the sum S - 1 of all but the
    first:   d log S = u (6 lead + 8 + links) (S - 1) / S.
    The spread is taken off sum e (z - ref) = spread + lead (S - 1) at most, as a difference of two such sums, each with that error and 2 u for
    its products and the last addition:   d = 2 u (6 lead + 12 + links) (spread + lead (S - 1)) / S."""
    ref = _reference(z, tokens, n)
    u, links = 2.0 ** -24, z.shape[1] / 256 + 64
    d = z.max(1, keepdim=True).values - z
    e = torch.exp(-d)
    S, spread = e.sum(1), (e * d).sum(1)
    d_log = u * (6 * lead + 8 + links) * (S - 1) / S
    d_spread = 2 * u * (6 * lead + 12 + links) * (spread + lead * (S - 1)) / S
    more = {"token_logp": d_log[:, None], "entropy": d_log + d_spread, "conf": d_log / S, "top_idx": None, "top_logp": d_log[:, None]}
    return {k: (v, None if err is None else err + more[k]) for k, (v, err) in ref.items()}


@pytest.mark.parametrize("T, V", [(1, 131072), (8, 131072), (64, 60001), (300, 9000), (700, 20000), (2600, 5000)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_late_plateaus(T, V, dtype):
    """A first part of every share of the row 1 to just below 20 under a long plateau; a plateau in the last entries alone; one of two entries."""
    z = torch.empty((T, V))
    for t in range(T):
        under = (1.0, 7.25, 13.0, 19.0, 19.875)[t % 5]
        first = V - 3 if t % 3 == 1 else max(V // 3, 1)
        z[t, :first], z[t, first:] = 4.0 - under, 4.0
        if t % 3 == 2:
            z[t, first + 2:] = 4.0 - under
    z = z.to(dtype)
    tokens = _tokens(T, 2, V, T)
    tokens[:, 0] = V - 2
    b = mm.LogprobBuffers(T, 2, 9, V).run(z.cuda(), tokens.cuda())
    for name, (want, err) in _wider(z.double(), tokens, 9, LEAD).items():
        got = getattr(b, name).cpu()
        assert torch.equal(got.long(), want) if err is None else bool(((got.double() - want).abs() <= err).all()), name
