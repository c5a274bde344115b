"""Rows of larger tensors: the last positions of a batch of prompts, as tokens of a projection and as logits."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("B, S, K, dtype", [(3, 1024, 4096, BF16), (40, 1025, 4099, BF16), (70, 1100, 4096, FP32), (1, 2000, 4096, FP32), (5, 1030, 4096, FP32)])
def test_last_hidden_states_of_a_batch(B, S, K, dtype):
    """Quantised by the product's own workgroups, in front of the streaming kernel and in front of tiles."""
    hidden = torch.zeros((B, S, K), dtype=dtype, device="cuda")
    hidden[:, -1] = torch.randn((B, K), generator=_gen(B)).to(dtype).cuda()
    x = hidden[:, -1]
    assert B == 1 or x.stride(0) >= 1 << 22
    lin = mm.Int8Linear.quantize(torch.randn((300, K), generator=_gen(1)).cuda())
    assert torch.equal(lin(x), lin(x.contiguous()))
    for got, want in zip(mm.quantize_rows(x), mm.quantize_rows(x.contiguous())):
        assert torch.equal(got, want)


@pytest.mark.parametrize("B, S, V, dtype", [(3, 40, 131072, BF16), (1, 40, 131072, FP32), (300, 70, 65537, BF16)])
def test_last_logits_of_a_batch(B, S, V, dtype):
    logits = torch.zeros((B, S, V), dtype=dtype, device="cuda")
    logits[:, -1] = (torch.randn((B, V), generator=_gen(V)) * 3).to(dtype).cuda()
    z = logits[:, -1]
    assert B == 1 or z.stride(0) >= 1 << 22
    got, want = mm.LogprobBuffers(B, 0, 7, V).run(z), mm.LogprobBuffers(B, 0, 7, V).run(z.contiguous())
    for name in ("entropy", "conf", "top_idx", "top_logp"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name
