"""The 8-bit product at the sizes that choose each of its kernels, tile heights and edges, against 64 bits."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from test_gpu_output_head import BF16, FP32, _bound, _gen, _operands, _product, _run_codes

pytestmark = pytest.mark.gpu

# large outputs: last tiles of one row and one column, K below, at and behind the vector, the chunk and the ring.  Most of these sizes run on tiles of
# 64 x 64 in two stages, four on those of 128, 192 or 256 x 256, which test_gpu_int8_routes.py has by kernel
WIDE = [(65, 33000, 77), (97, 32800, 16), (128, 33025, 400), (129, 32769, 33), (192, 33000, 129), (193, 32770, 1000), (256, 33000, 7), (257, 16640, 128),
        (300, 20000, 1000), (513, 11009, 640), (700, 12000, 15), (2049, 20001, 200), (1100, 16384, 2000), (640, 9000, 385)]
# few outputs or tokens: tiles of 64 x 64
TILE = [(65, 128, 128), (65, 1, 1), (127, 129, 255), (128, 1000, 2048), (130, 127, 384), (191, 640, 100), (333, 2000, 1111), (700, 2048, 512), (1000, 130, 4097),
        (4096, 129, 64)]
# up to 64 tokens: 1 to 4 blocks of 16, K split over waves or not, the last step whole, in part and alone
STREAM = [(1, 16, 64), (1, 70000, 48), (5, 500, 63), (15, 1000, 4096), (16, 66001, 128), (17, 65600, 100), (31, 17, 700), (32, 3000, 2000), (33, 66000, 320),
          (47, 999, 511), (48, 1024, 513), (49, 65700, 65), (63, 100, 8191), (64, 131072, 257)]


@pytest.mark.parametrize("T, N, K", WIDE + TILE + STREAM)
@pytest.mark.parametrize("dtype, with_bias", [(FP32, True), (BF16, False)])
def test_product_of_codes(T, N, K, dtype, with_bias):
    x, w, xs, ws, bias = _operands(T, N, K, seed=T + 3 * N + 7 * K)
    ref, part = _product(x, w, xs, ws, bias if with_bias else None, K)
    got = _run_codes(x.cuda(), w.cuda(), xs.cuda(), ws.cuda(), bias.cuda() if with_bias else None, K, dtype, N + 5 if with_bias else None)
    assert ((got.cpu().double() - ref).abs() <= _bound(ref, part, dtype)).all()


# tiles of 64 x 64 (a CU each, or two to a CU) and of 64 x 128, with K shared by two groups of waves or not; K below, at and behind the chunk, the ring
# and what each group gets; last tiles of one row and one column; up to 64 tokens whose K is too long for the streaming kernel
SMALL_TILES = [(65, 64, 128), (66, 65, 1024), (128, 1000, 1536), (193, 2050, 1537), (65, 1000, 1600), (257, 127, 2049), (300, 500, 4000), (1, 100, 20000), (33, 300, 5001),
               (300, 4000, 500), (333, 5000, 1000), (129, 8001, 1535), (333, 5000, 1700), (129, 8065, 1541), (449, 4097, 2300), (64, 16385, 4200),
               (333, 7000, 1111), (65, 32801, 99), (1000, 4100, 2500), (2000, 1030, 1552)]

# more tiles than can be under way at once, short K: two stages
SMALL_TILES += [(300, 16400, 77), (65, 40001, 128), (130, 33000, 300), (700, 7001, 513), (129, 22000, 640), (2049, 2700, 16), (100, 50000, 7)]

@pytest.mark.parametrize("T, N, K", SMALL_TILES)
@pytest.mark.parametrize("dtype, with_bias", [(FP32, False), (BF16, True)])
def test_product_on_small_tiles(T, N, K, dtype, with_bias):
    test_product_of_codes(T, N, K, dtype, with_bias)


@pytest.mark.parametrize("T, K", [(1, 1), (1, 700), (1, 16384), (2, 8192), (3, 33), (3, 5461), (4, 1000), (7, 2340), (8, 64), (8, 2048), (15, 1092), (16, 5), (16, 1024),
                                  (16, 1025), (17, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("N", [40, 66000])
def test_small_batches_of_floats_are_the_two_calls(T, K, dtype, N):
    """Tokens that the product's own workgroups quantise, at any alignment, rows without numbers and of zeros among them."""
    mem = (torch.randn((T * (K + 3) + 1,), generator=_gen(T + K)) * 3).to(dtype).cuda()
    x = mem.as_strided((T, K), (K + 3, 1), 1)
    if T > 2:
        x[1], x[2, K // 2] = 0.0, float("inf")
    g = torch.Generator(device="cuda").manual_seed(K)
    w = torch.randint(-128, 128, (N, (K + 15) // 16 * 16), generator=g, device="cuda").to(torch.int8)
    lin = mm.Int8Linear(w[:, :K], torch.rand((N,), generator=g, device="cuda"), torch.randn((N,), generator=g, device="cuda"))
    got = lin(x)
    q, s = mm.quantize_rows(x)
    want = lin(q, x_scale=s)
    assert torch.equal(got.nan_to_num(7e9), want.nan_to_num(7e9))
    if T > 2:
        assert torch.equal(got[1], lin.bias) and got[2].isnan().all() and got.isnan().sum() == N


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows, K", [(700, 100), (5, 1024), (5, 1025), (3, 2048), (3, 2049), (9, 4096), (2, 8193), (2, 40000), (1, 131071)])
def test_scales_and_codes_of_long_rows(rows, K, dtype):
    """64 bits decide every code: near a tie 127 x / a is a whole multiple of 2^-33 away from it, or on it."""
    x = (torch.randn((rows, K), generator=_gen(K)) * torch.exp(torch.randn((rows, 1), generator=_gen(rows)))).to(dtype)
    q, s = mm.quantize_rows(x.cuda())
    a = x.double().abs().amax(1, keepdim=True)
    assert torch.equal(s.cpu(), (a.float() / 127.0).reshape(-1))
    assert torch.equal(q.cpu().double(), (127.0 * x.double() / a).round())
