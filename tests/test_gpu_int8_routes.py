"""The 8-bit product on every kernel and tile at their edges, against 64 bits, and the same bits on all of them.  Which kernel a size takes is asserted
in test_int8_route_host.py."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from test_gpu_output_head import BF16, FP32, _bound, _operands, _product, _run_codes

pytestmark = pytest.mark.gpu

# Per kernel: codes below a vector of 16, below and above three chunks with a rest behind the last vector, ragged in both directions; whole tiles;
# K whole vectors but no whole chunk; more tiles than workgroups (wide), many tokens.
ROUTES = {
    "wide2": [(453, 47477, 4), (323, 40707, 134), (70, 34611, 1091), (128, 33024, 1152), (127, 32769, 656), (2350, 6541, 131)],
    "wide3": [(325, 56219, 3), (333, 29919, 133), (134, 46013, 1049), (192, 43776, 768), (384, 32768, 768), (191, 44033, 656), (2131, 5281, 129)],
    "wide4": [(198, 60847, 14), (395, 30039, 130), (193, 33565, 1043), (256, 33024, 1152), (193, 33536, 1040), (2049, 20001, 97), (1873, 6965, 131)],
    "k128": [(269, 51761, 6), (294, 39201, 134), (72, 24849, 1001), (128, 16512, 2304), (65, 24833, 1040), (2507, 6481, 130)],
    "k128Shared": [(66, 8297, 1729), (128, 8320, 1792), (131, 8193, 5003), (64, 16512, 4224), (449, 2049, 1552)],
    "k64Shared": [(67, 71, 1593), (128, 4096, 2048), (65, 1000, 5001), (1000, 1001, 1552), (33, 129, 4999)],
    "k64": [(67, 71, 1), (65, 77, 142), (66, 77, 1074), (128, 8192, 1024), (2999, 129, 600), (300, 8001, 1900)],
    "k64Short": [(65, 24881, 7), (66, 25571, 182), (81, 24961, 145), (128, 33024, 384), (2500, 1281, 636), (130, 25001, 336)],
}

# Of one product of 800 x 40000, rows and columns that take other kernels: a part's bits are those of the whole.
WHOLE = (800, 40000)
PARTS = {
    1723: [(0, 800, 0, 40000), (1, 2, 5, 39000), (3, 67, 0, 40000), (7, 73, 100, 8397), (0, 65, 3, 75), (100, 300, 0, 10000), (20, 92, 0, 24848), (0, 333, 0, 40000),
           (411, 800, 9, 20001), (0, 130, 77, 39999), (600, 800, 1000, 35000), (5, 138, 0, 40000), (0, 70, 2000, 37000)],
    601: [(0, 800, 0, 40000), (2, 60, 0, 40000), (0, 65, 5, 33000), (100, 171, 3, 75), (0, 450, 0, 40000), (300, 633, 7, 29007), (1, 396, 0, 30039), (64, 192, 0, 33024)],
}


@pytest.mark.parametrize("T, N, K", [s for sizes in ROUTES.values() for s in sizes])
@pytest.mark.parametrize("dtype, with_bias", [(FP32, True), (BF16, False)])
def test_product_on_every_kernel(T, N, K, dtype, with_bias):
    x, w, xs, ws, bias = _operands(T, N, K, seed=3 * T + N + 11 * K)
    ref, part = _product(x, w, xs, ws, bias if with_bias else None, K)
    got = _run_codes(x.cuda(), w.cuda(), xs.cuda(), ws.cuda(), bias.cuda() if with_bias else None, K, dtype, N + 3 if with_bias else None)
    assert ((got.cpu().double() - ref).abs() <= _bound(ref, part, dtype)).all()


@pytest.mark.parametrize("K", PARTS)
def test_every_kernel_gives_the_same_bits(K):
    x, w, xs, ws, bias = [t.cuda() for t in _operands(*WHOLE, K, seed=K)]
    whole = _run_codes(x, w, xs, ws, bias, K, FP32)
    assert torch.equal(_run_codes(x, w, xs, ws, bias, K, BF16), whole.to(BF16))
    for t0, t1, n0, n1 in PARTS[K]:
        args = x[t0:t1], w[n0:n1], xs[t0:t1].clone(), ws[n0:n1].clone(), bias[n0:n1].clone(), K
        assert torch.equal(_run_codes(*args, FP32), whole[t0:t1, n0:n1]), (t0, t1, n0, n1)
        assert torch.equal(_run_codes(*args, BF16), whole[t0:t1, n0:n1].to(BF16)), (t0, t1, n0, n1)
