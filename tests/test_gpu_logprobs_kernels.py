"""Log probabilities at the sizes that choose each split of a row, and on rows made to go wrong there, against 64 bits."""
import math

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from test_gpu_output_head import BF16, FP32, _check_logprobs, _gen, _tokens

pytestmark = pytest.mark.gpu


# a wave per row; four waves; eight waves and 1 to 16 workgroups
@pytest.mark.parametrize("T, V", [(2048, 3000), (2100, 9001), (500, 20003), (400, 8192), (1000, 5119), (256, 50000), (100, 131071), (33, 160001), (9, 70007), (2, 159999),
                                  (1, 16384), (64, 17000)])
@pytest.mark.parametrize("dtype, n_top", [(FP32, 20), (BF16, 7)])
def test_splits_of_a_row(T, V, dtype, n_top):
    z = torch.randn((T, V), generator=_gen(V)) * 3.0
    hot = torch.randint(0, V, (T,), generator=_gen(T))
    z[torch.arange(T), hot] += torch.rand((T,), generator=_gen(T + 1)) * 25
    _check_logprobs(z.to(dtype), _tokens(T, 2, V, T), n_top)


# two, four, eight and sixteen workgroups a row, at the lengths where they begin
@pytest.mark.parametrize("T, V", [(128, 64513), (64, 48129), (63, 50001), (32, 72705), (20, 80001), (16, 261121), (3, 270001)])
@pytest.mark.parametrize("dtype, n_top", [(FP32, 5), (BF16, 1)])
def test_parts_of_a_row(T, V, dtype, n_top):
    test_splits_of_a_row(T, V, dtype, n_top)


@pytest.mark.parametrize("T, V", [(1, 131072), (5, 40000), (300, 9000), (450, 4100), (2050, 2100)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_rows_in_order_and_in_steps(T, V, dtype):
    """Rising rows (every batch changes the list), falling ones, a single step at the end, equal entries but for one, in every split."""
    k = torch.arange(V).float()
    z = torch.zeros((T, V))
    rows = [k / V * 30, -k / V * 30, (k // 997).remainder(13), torch.where(k == V - 1, 9.0, 0.0), torch.full((V,), -2.5)]
    for t in range(T):
        z[t] = rows[t % 5] + (t // 5) * 0.125
    _check_logprobs(z.to(dtype), _tokens(T, 1, V, T), 32)


@pytest.mark.parametrize("T, V", [(1, 60000), (3, 131072), (420, 5000), (2060, 1500)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_rows_of_far_numbers(T, V, dtype):
    """Offsets of a million, the type's largest and lowest numbers, entries that are nothing beside the largest, in one row and in one wave's
    share of it only."""
    big = torch.finfo(dtype).max
    base = torch.randn((T, V), generator=_gen(V)) * 3.0
    z = base.clone()
    for t in range(T):
        kind = t % 6 if T > 6 else (t + 1)
        if kind == 1:
            z[t] += 1.0e6
        elif kind == 2:
            z[t, V // 2:] = -big
        elif kind == 3:
            z[t] = -big
            z[t, ::3] = -big / 2
        elif kind == 4:
            z[t, V // 3] = big
        elif kind == 5:
            z[t, : V // 2] -= 5000.0
    # a million in bf16 has steps of 8192 and in fp32 of 1/16: what counts are the stored numbers
    _check_logprobs(z.to(dtype), _tokens(T, 3, V, V), 16)


@pytest.mark.parametrize("T, V", [(1, 131072), (40, 30000), (500, 9000), (2048, 2500)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_rows_with_few_tokens_left(T, V, dtype):
    """Fewer entries than alternatives, anywhere in the row, the others -inf."""
    z = torch.full((T, V), -math.inf)
    for t in range(T):
        n = 1 + t % 23
        at = torch.randint(0, V, (n,), generator=_gen(t))
        z[t, at] = torch.randn((n,), generator=_gen(t + 1)).to(dtype).float() * 5
    _check_logprobs(z.to(dtype), _tokens(T, 1, V, T), 20)


@pytest.mark.parametrize("bits", [0x7fc1, 0xffc0, 0x7f81, 0xff81, 0x7fff])
@pytest.mark.parametrize("V, T", [(3000, 2), (131072, 1), (9000, 450), (2000, 2050)])
def test_nan_of_every_sign_and_kind(bits, V, T):
    """Quiet and signalling NaN of either sign take every number of their row; order and the other rows are as without them."""
    z = (torch.randn((T, V), generator=_gen(V)) * 3).to(BF16)
    clean = z.clone()
    raw = z.view(torch.int16)
    at = [0, V // 2, V - 1]
    for i in at:
        raw[0, i] = bits - 65536 if bits > 32767 else bits
    b = mm.LogprobBuffers(T, 1, 9, V).run(z.cuda(), _tokens(T, 1, V, 1).cuda())
    assert b.entropy[0].isnan() and b.conf[0].isnan() and b.top_logp[0].isnan().all() and b.token_logp[0].isnan().all()
    clean[0, at] = -math.inf
    order = torch.sort(clean.float(), dim=1, descending=True, stable=True).indices[:, :9]
    assert torch.equal(b.top_idx.cpu().long(), order)
    if T > 1:
        assert not (b.entropy[1:].isnan().any() or b.conf[1:].isnan().any() or b.top_logp[1:].isnan().any())


@pytest.mark.parametrize("T, V, dtype", [(300, 9000, BF16), (1100, 9000, FP32), (2100, 2500, BF16), (2100, 1300, FP32), (64, 40000, FP32), (128, 70000, BF16)])
def test_signalling_nan_beside_the_best_tokens(T, V, dtype):
    """In every place of a lane's entries, in front of and behind tokens that belong to the list."""
    z = (torch.randn((T, V), generator=_gen(V)) * 3).to(dtype)
    rows = torch.arange(T)
    at = (rows * 37) % V
    for step in (1, 3, 5):
        z[rows, (at + step) % V] = 30.0 + step
    clean = z.clone()
    clean[rows, at] = clean[rows, (at + 4) % V] = -math.inf
    raw, bits = (z.view(torch.int16), 0x7f81) if dtype is BF16 else (z.view(torch.int32), 0x7f800001)
    raw[rows, at] = bits
    raw[rows, (at + 4) % V] = bits
    b = mm.LogprobBuffers(T, 0, 12, V).run(z.cuda())
    assert b.conf.isnan().all() and b.entropy.isnan().all()
    order = torch.sort(clean.float(), dim=1, descending=True, stable=True).indices[:, :12]
    assert torch.equal(b.top_idx.cpu().long(), order)


def test_a_row_has_the_same_bits_in_every_call():
    """The order of the sums does not depend on which wave comes first."""
    for T, V, dtype in ((1, 131072, BF16), (37, 50257, FP32), (500, 20000, BF16), (2048, 3001, FP32)):
        z = (torch.randn((T, V), generator=_gen(T)) * 4).to(dtype).cuda()
        tokens = _tokens(T, 2, V, 1).cuda()
        first = mm.LogprobBuffers(T, 2, 11, V).run(z, tokens)
        for _ in range(5):
            b = mm.LogprobBuffers(T, 2, 11, V).run(z, tokens)
            for name in ("token_logp", "entropy", "conf", "top_idx", "top_logp"):
                assert torch.equal(getattr(b, name), getattr(first, name)), (T, name)


def test_workspace_of_more_than_one_workgroup_per_row():
    """A workspace that holds anything, and one that a larger call has used."""
    T, V = 3, 131072
    z = (torch.randn((T, V), generator=_gen(0)) * 4).cuda()
    want = mm.LogprobBuffers(T, 0, 5, V).run(z)
    b = mm.LogprobBuffers(T, 0, 5, V)
    assert b.ws.numel() > 0
    for fill in (0xff, 0x7f, 0):
        b.ws.fill_(fill)
        b.run(z)
        assert torch.equal(b.top_idx, want.top_idx) and torch.equal(b.top_logp, want.top_logp) and torch.equal(b.entropy, want.entropy)
