"""The output head's calls with one tensor of another device among the right ones: refused before anything is enqueued."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.gpu


def test_one_host_tensor_among_device_tensors():
    w = torch.ones((8, 64), dtype=torch.int8, device="cuda")
    lin = mm.Int8Linear(w, torch.ones(8, device="cuda"))
    codes, x, scale = w[:2], torch.ones((2, 64), device="cuda"), torch.ones(2, device="cuda")
    assert (lin(codes, x_scale=scale) == 64.0).all()
    for call in (lambda: lin(codes, x_scale=scale.cpu()), lambda: lin(x.cpu()), lambda: lin(codes.cpu(), x_scale=scale),
                 lambda: lin(x, out=torch.empty((2, 8)))):
        with pytest.raises(ValueError, match="device"):
            call()
    tokens = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    b = mm.LogprobBuffers(2, 1, 1, 64)
    assert (b.run(x, tokens).top_idx == 0).all()
    for z, t, buffers in ((x.cpu(), tokens, b), (x, tokens.cpu(), b), (x, tokens, mm.LogprobBuffers(2, 1, 1, 64, device="cpu"))):
        with pytest.raises(ValueError, match="device"):
            buffers.run(z, t)
    with pytest.raises(ValueError, match="given"):
        b.run(x)
    q, s = torch.empty((2, 64), dtype=torch.int8), torch.empty(2)
    for a in ((x, q.cuda(), s), (x, q, s.cuda()), (x.cpu(), q.cuda(), s.cuda())):
        with pytest.raises(ValueError, match="device"):
            mm.moe_quantize_rows(*a)
    with pytest.raises(ValueError, match="device"):
        mm.moe_matmul_int8(mm.int8_config(codes, w, x[:, :8]), codes, scale, w, lin.w_scale, torch.zeros(8), x[:, :8])
