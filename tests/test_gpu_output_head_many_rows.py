"""More rows than one launch of a workgroup per row may have (2^32 threads): short rows at places where a launch may end."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from test_gpu_output_head import _reference

pytestmark = pytest.mark.gpu
ROWS = 2 ** 26 + 5


def _places():
    """Rows at either end and around powers of two, where a launch may end and the next begin."""
    return torch.unique(torch.tensor([min(max(c + d, 0), ROWS - 1) for c in [0, ROWS] + [k * 2 ** e for e in (20, 22, 24) for k in (1, 2, 3, 4)] + [2 ** 26]
                                      for d in range(-3, 4)])).cuda()


def test_codes_of_many_rows():
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((ROWS, 3), generator=g, device="cuda", dtype=torch.bfloat16)
    q, s = mm.quantize_rows(x)
    at = _places()
    want = mm.quantize_rows(x[at])
    assert torch.equal(q[at], want[0]) and torch.equal(s[at], want[1])
    assert torch.equal(s.cpu(), x.abs().amax(1).float().cpu() / 127.0)      # on the host: a device's division by a number may be a product


def test_log_probabilities_of_many_rows():
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn((ROWS, 5), generator=g, device="cuda", dtype=torch.bfloat16)
    tokens = torch.randint(0, 5, (ROWS, 1), generator=g, device="cuda").to(torch.int32)
    b = mm.LogprobBuffers(ROWS, 1, 1, 5)
    for t in (b.token_logp, b.entropy, b.conf, b.top_logp, b.top_idx):
        t.fill_(7)                                            # no value of five tokens
    b.run(z, tokens)
    at = _places()
    # a row that starts elsewhere within 16 bytes may add its entries in another order, so the bounds are those of the definition
    for name, (want, err) in _reference(z[at].double().cpu(), tokens[at].cpu(), 1).items():
        got = getattr(b, name)[at].cpu()
        assert torch.equal(got.long(), want) if err is None else bool(((got.double() - want).abs() <= err).all()), name
        assert (getattr(b, name) != 7).all(), name


def test_a_projection_of_many_tokens():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((ROWS, 4), generator=g, device="cuda", dtype=torch.bfloat16)
    lin = mm.Int8Linear.quantize(torch.randn((2, 4), generator=g, device="cuda"))
    out = lin(x)
    at = _places()
    assert torch.equal(out[at], lin(x[at]))
