"""The output head's operators against their definitions in 64 bits: codes of rows, the 8-bit product, log probabilities."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}          # half a step of the type, relative to the value


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------ codes and scales
def _code(x, a):
    """Nearest integer to 127 x / a of the rationals, ties to even (Python's own rounding of a fraction)."""
    return round(Fraction(127) * Fraction(x) / Fraction(a)) if a else 0


def _check_codes(x, ldq=None, view=None):
    """x: CPU tensor [rows, K]; view: the device tensor holding it (default: a dense copy)."""
    rows, K = x.shape
    ldq = (K + 15) // 16 * 16 if ldq is None else ldq
    q = torch.full((rows + 1, ldq), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((rows + 1,), 5.0, dtype=FP32, device="cuda")
    mm.moe_quantize_rows(x.cuda() if view is None else view, q[:rows], scale[:rows])
    q, scale = q.cpu(), scale.cpu()
    assert (q[rows] == 77).all() and scale[rows] == 5.0
    assert (q[:rows, K:] == 0).all()
    for r in range(rows):
        v = x[r].double().numpy()
        if not np.isfinite(v).all():
            assert math.isnan(scale[r]) and (q[r] == 0).all()
            continue
        a = np.abs(v).max()
        assert scale[r].item() == np.float32(a) / np.float32(127.0)
        assert q[r, :K].tolist() == [_code(e, a) for e in v.tolist()], r


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows, K", [(1, 1), (3, 2), (2, 15), (5, 16), (2, 17), (3, 255), (2, 256), (2, 1971), (1, 4096), (1, 8200), (300, 33)])
def test_codes(dtype, rows, K):
    x = torch.randn((rows, K), generator=_gen(K)) * torch.exp(2 * torch.randn((rows, 1), generator=_gen(rows)))
    _check_codes(x.to(dtype))


def test_codes_at_ties_and_next_to_them():
    """Largest magnitude 254: every odd integer is a tie (127 x / 254 = x / 2).  fp32 neighbours of the ties fall to either side."""
    odd = torch.arange(-253, 254, 2).float()
    x = torch.cat([torch.tensor([254.0]), odd]).reshape(1, -1)
    _check_codes(x)
    _check_codes(x.to(BF16))
    up, down = torch.nextafter(odd, torch.tensor(math.inf)), torch.nextafter(odd, torch.tensor(-math.inf))
    _check_codes(torch.cat([torch.tensor([-254.0]), up, down]).reshape(1, -1))
    # ties under other magnitudes: x = (2 n + 1) a / 254 is a number for a = 127 2^j
    for j in (-140, -120, -30, 60, 121):
        a = 127.0 * 2.0 ** j
        x = torch.tensor([[a] + [(2 * n + 1) / 2.0 * 2.0 ** j for n in range(0, 127, 5)]], dtype=FP32)
        _check_codes(torch.cat([x, torch.nextafter(x[:, 1:], torch.tensor(math.inf))], dim=1))


def test_codes_of_special_rows():
    big, tiny = torch.finfo(FP32).max, 2.0 ** -149
    x = torch.zeros((9, 40))
    x[1, 3] = -0.0
    x[2, 7], x[2, 8], x[2, 9] = big, -big, big / 254
    x[3, 0], x[3, 39], x[3, 5] = tiny, -tiny, 0.0
    x[4, 1], x[4, 2], x[4, 3] = 300 * tiny, 150 * tiny, -7 * tiny
    x[5, 11] = math.nan
    x[6, 39], x[6, 0] = math.inf, 1.0
    x[7, 0] = -math.inf
    x[8, 17] = 2.0 ** -126
    _check_codes(x)
    _check_codes(x[[0, 1, 5, 6, 7, 8]].to(BF16))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_codes_of_strided_rows_at_any_alignment(dtype):
    for K, ld, first in ((100, 103, 1), (64, 64, 3), (1000, 1001, 5), (4099, 4111, 7)):
        mem = torch.randn((first + 4 * ld,), generator=_gen(K)).to(dtype)
        dev = mem.cuda()
        x = mem[first:].as_strided((4, K), (ld, 1), first)
        _check_codes(x, ldq=(K + 15) // 16 * 16 + 32, view=dev.as_strided((4, K), (ld, 1), first))


# ------------------------------------------------------------------------------------ product
def _operands(T, N, K, seed, extremes=False):
    g = _gen(seed)
    pad = (K + 15) // 16 * 16
    # what stands behind K must not matter
    x = torch.randint(-128, 128, (T, pad + 16), generator=g).to(torch.int8)
    w = torch.randint(-128, 128, (N, pad + 32), generator=g).to(torch.int8)
    if extremes:
        x[:, :K], w[:, :K] = -128, -128
        w[N // 2, :K] = 127
    return (x, w, torch.rand((T,), generator=g) * 0.1 + 1e-3, torch.rand((N,), generator=g) * 0.1 + 1e-3, torch.randn((N,), generator=g) * 10)


def _product(x, w, xs, ws, bias, K):
    """-> (value, size of the part that rounds three times), in 64 bits."""
    p = (x[:, :K].double() @ w[:, :K].double().t().contiguous()) * xs.double()[:, None] * ws.double()[None, :]
    return (p if bias is None else p + bias.double()), p.abs()


def _bound(ref, part, dtype):
    """The sum to fp32 and two products by scales, half a step each of the part without the bias; with the bias one more of the
    result; the output type's own."""
    return part * (3 * 2.0 ** -24) * 1.0001 + ref.abs() * (2.0 ** -24 + (HALF[BF16] * 1.0001 if dtype == BF16 else 0.0))


def _run_codes(x, w, xs, ws, bias, K, dtype, ldo=None):
    T, N = x.shape[0], w.shape[0]
    ldo = N if ldo is None else ldo
    out = torch.full((T + 1, ldo), 3.0, dtype=dtype, device="cuda")
    c = mm.int8_config(x[:, :K], w[:, :K], out[:T, :N])
    mm.moe_matmul_int8(c, x[:, :K], xs, w[:, :K], ws, bias, out[:T, :N])
    assert (out[T] == 3.0).all() and (out[:, N:] == 3.0).all()
    return out[:T, :N]


SHAPES = [(1, 1, 1), (1, 1, 16), (2, 3, 5), (1, 33, 64), (1, 2048, 2048), (3, 100, 17), (7, 65, 1000), (8, 640, 512), (16, 257, 31), (17, 128, 300),
          (31, 129, 96), (33, 1000, 127), (64, 500, 2049), (65, 64, 64), (100, 777, 255), (128, 256, 128), (129, 257, 129), (200, 512, 144),
          (255, 130, 640), (256, 256, 1024), (300, 1000, 200), (513, 384, 2000), (700, 2048, 333), (1030, 300, 65)]


@pytest.mark.parametrize("T, N, K", SHAPES)
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_product(T, N, K, dtype):
    x, w, xs, ws, bias = _operands(T, N, K, seed=T * 7919 + N + K)
    d = [t.cuda() for t in (x, w, xs, ws, bias)]
    for with_bias, ldo in ((False, N), (True, N + 3)):
        ref, part = _product(x, w, xs, ws, bias if with_bias else None, K)
        got = _run_codes(*d[:4], d[4] if with_bias else None, K, dtype, ldo).cpu().double()
        assert ((got - ref).abs() <= _bound(ref, part, dtype)).all(), ((got - ref).abs() - _bound(ref, part, dtype)).max()


@pytest.mark.parametrize("T", [2, 40, 300])
def test_product_of_the_largest_sums(T):
    """K at its limit, every code -128: the sums reach 2^31 - 2^14."""
    K, N = mm.MOE_INT8_MAX_K, 40
    x, w, xs, ws, _ = _operands(T, N, K, seed=T, extremes=True)
    ref, part = _product(x, w, xs, ws, None, K)
    got = _run_codes(x.cuda(), w.cuda(), xs.cuda(), ws.cuda(), None, K, FP32).cpu().double()
    assert ((got - ref).abs() <= _bound(ref, part, FP32)).all()


def test_an_output_has_the_same_bits_whatever_else_is_computed():
    """Sizes of every kernel and tile against slices of one large product."""
    T, N, K = 700, 2100, 1000
    x, w, xs, ws, bias = [t.cuda() for t in _operands(T, N, K, seed=5)]
    whole = _run_codes(x, w, xs, ws, bias, K, FP32)
    half = _run_codes(x, w, xs, ws, bias, K, BF16)
    assert torch.equal(whole.to(BF16), half)
    for t0, t1, n0, n1 in ((0, 1, 0, N), (699, 700, 3, 400), (5, 13, 0, N), (20, 52, 100, 164), (0, 64, 0, N), (1, 66, 0, N), (100, 228, 0, 1000),
                           (0, 130, 77, 2100), (300, 556, 0, 512), (44, 700, 9, 2000), (0, 333, 0, 333)):
        got = _run_codes(x[t0:t1], w[n0:n1], xs[t0:t1].clone(), ws[n0:n1].clone(), bias[n0:n1].clone(), K, FP32)
        assert torch.equal(got, whole[t0:t1, n0:n1]), (t0, t1, n0, n1)


def test_product_with_broken_and_empty_rows():
    """A token with scale NaN gives NaN, one with scale 0 the bias; the rows beside them are untouched."""
    x, w, xs, ws, bias = [t.cuda() for t in _operands(20, 100, 64, seed=3)]
    good = _run_codes(x, w, xs, ws, bias, 64, FP32)
    xs[3], xs[7] = math.nan, 0.0
    got = _run_codes(x, w, xs, ws, bias, 64, FP32)
    assert got[3].isnan().all() and torch.equal(got[7], bias)
    keep = [t for t in range(20) if t not in (3, 7)]
    assert torch.equal(got[keep], good[keep])


@pytest.mark.parametrize("T", [1, 4, 9, 64, 130, 600])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_linear_is_the_two_calls(T, dtype):
    N, K = 300, 1971
    x = (torch.randn((T, K), generator=_gen(T)) * 3).to(dtype).cuda()
    x[T // 2, 5] = math.nan
    weight = torch.randn((N, K), generator=_gen(T + 1)).cuda()
    lin = mm.Int8Linear.quantize(weight, torch.randn((N,), generator=_gen(T + 2)).cuda())
    q, s = mm.quantize_rows(x)
    for out_type in (BF16, FP32):
        got = lin(x, out=torch.empty((T, N), dtype=out_type, device="cuda"))
        want = lin(q, x_scale=s, out=torch.empty((T, N), dtype=out_type, device="cuda"))
        assert torch.equal(got.nan_to_num(7e9), want.nan_to_num(7e9)) and got[T // 2].isnan().all() and got.isnan().sum() == N
    # close to the float product: each operand's step is a / 127, errors up to half a step, independent, over K terms
    ok = [t for t in range(T) if t != T // 2]
    if ok:
        f = x.double().cpu()[ok] @ weight.double().cpu().t() + lin.bias.double().cpu()
        step_x, step_w = s.double().cpu()[ok], lin.w_scale.double().cpu()
        rms = ((step_x[:, None] ** 2 * (weight.double().cpu() ** 2).sum(1)[None, :] + step_w[None, :] ** 2 * (x.double().cpu()[ok] ** 2).sum(1)[:, None]) / 12).sqrt()
        assert ((lin(x).cpu().double()[ok] - f).abs() <= 7 * rms).all()


def test_linear_of_strided_tokens_on_another_stream():
    T, N, K, ld = 50, 200, 333, 341
    mem = torch.randn((T * ld + 1,), generator=_gen(0)).to(BF16).cuda()
    x = mem.as_strided((T, K), (ld, 1), 1)
    lin = mm.Int8Linear.quantize(torch.randn((N, K), generator=_gen(1)).cuda())
    want = lin(x.contiguous())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lin(x, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_products_with_no_tokens():
    lin = mm.Int8Linear.quantize(torch.randn((30, 48), generator=_gen(1)).cuda())
    assert lin(torch.empty((0, 48), device="cuda")).shape == (0, 30)


def test_product_and_logprobs_in_a_graph():
    """One captured step (hidden states to alternatives), replayed on new inputs between eager calls."""
    T, N, K = 9, 5000, 256
    lin = mm.Int8Linear.quantize(torch.randn((N, K), generator=_gen(1)).cuda())
    b, b2 = mm.LogprobBuffers(T, 2, 5, N), mm.LogprobBuffers(T, 2, 5, N)
    x = torch.zeros((T, K), dtype=BF16, device="cuda")
    tokens = torch.randint(0, N, (T, 2), generator=_gen(2)).to(torch.int32).cuda()
    out = torch.empty((T, N), dtype=FP32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run(lin(x, out=out), tokens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(lin(x, out=out), tokens)
    lin2 = mm.Int8Linear(lin.w, lin.w_scale)
    for i in range(4):
        x.copy_(torch.randn((T, K), generator=_gen(10 + i)).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        b2.run(lin2(x), tokens)
        torch.cuda.synchronize()
        for name in ("token_logp", "entropy", "conf", "top_idx", "top_logp"):
            assert torch.equal(getattr(b, name), getattr(b2, name)), (i, name)


# ------------------------------------------------------------------------------------ log probabilities
def _reference(z, tokens, n_top):
    """z: [T, V] float64 CPU, rows with a distribution.  -> dict of values and their error bounds.

    Bounds, u = 2^-24 (half an fp32 step).  A term e = exp(-d) of the sum beside the largest entry is off by u (difference) and
    2 u (product with log2 e) times d, and by 2 u of the exponential; the chains of additions, rescalings among them,
    have at most V / 256 + 64 links.  So the sum is off by at most r = u ((3 D + 2) + V / 256 + 64), D = sum e d / sum e, and
    log S by r times the sum's share of S, with 4 u of itself for the logarithm.  The spread sum e d has the same with D2 =
    sum e d^2 / sum e d, and 2 u for its products."""
    T, V = z.shape
    u = 2.0 ** -24
    m = z.max(1, keepdim=True).values
    d = m - z
    e = torch.exp(-d)
    first = z == m
    count = first.sum(1, keepdim=True).double()
    rest = torch.where(first, 0.0, e).sum(1, keepdim=True)
    S = count + rest
    log_s = torch.log(count) + torch.log1p(rest / count)
    ed = torch.where(e > 0, e * d, 0.0)
    ed2 = torch.where(e > 0, e * d * d, 0.0).sum(1, keepdim=True)
    spread = ed.sum(1, keepdim=True)
    tiny = 1e-300
    links = V / 256 + 64
    rel = u * (3 * spread / (rest + tiny) + 2 + links)
    d_log = rel * rest / S + 4 * u * log_s
    d_spread = spread / S * (u * (3 * ed2 / (spread + tiny) + 6 + links) + rel * rest / S + 2 * u)
    ent = log_s + spread / S
    lp = lambda v: (v - m) - log_s                                # noqa: E731
    lp_err = lambda v: u * (m - v) + d_log + u * lp(v).abs()      # noqa: E731
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :n_top]
    top = z.gather(1, order)
    t = tokens.long().clamp(0, V - 1)
    given = z.gather(1, t)
    pad = (tokens < 0) | (tokens >= V)
    return {"token_logp": (torch.where(pad, 0.0, lp(given)), torch.where(pad, 0.0, lp_err(given))),
            "entropy": (ent[:, 0], (d_log + d_spread + u * ent)[:, 0]),
            "conf": (1 / S[:, 0], ((rel * rest / S + 3 * u) / S)[:, 0]),
            "top_idx": (order, None), "top_logp": (lp(top), lp_err(top))}


def _check_logprobs(logits, tokens, n_top, rows=None, view=None):
    """logits, tokens on the CPU; view: the device tensor with the logits; rows: those with a distribution (default all)."""
    T, V = logits.shape
    b = mm.LogprobBuffers(T, tokens.shape[1], n_top, V)
    for t in (b.token_logp, b.entropy, b.conf, b.top_logp, b.top_idx):
        t.fill_(-5)
    b.run(logits.cuda() if view is None else view, tokens.cuda())
    rows = list(range(T)) if rows is None else rows
    ref = _reference(logits[rows].double(), tokens[rows], n_top)
    for name, (want, err) in ref.items():
        got = getattr(b, name).cpu()[rows]
        if err is None:
            assert torch.equal(got.long(), want), name
            continue
        got = got.double()
        inf = want.isinf()
        assert torch.equal(got[inf], want[inf]), name
        bad = ~((got - want).abs() <= err + 1e-44) & ~inf
        assert not bad.any(), (name, bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist(), err[bad][:3].tolist())
    return b


def _tokens(T, n, V, seed):
    return torch.randint(0, V, (T, n), generator=_gen(seed)).to(torch.int32)


LENGTHS = [1, 2, 7, 8, 63, 64, 65, 500, 511, 512, 513, 1000, 2047, 2048, 2049, 4097, 8192, 10007, 32000, 50257, 131073]


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("V", LENGTHS)
def test_logprobs_of_row_lengths(V, dtype):
    """Spread, confident and nearly uniform rows at every alignment (odd lengths), ties everywhere in bf16."""
    T = 6
    z = torch.randn((T, V), generator=_gen(V)) * 3.0
    z[1, V // 3] += 16.0
    z[2, V - 1] += 40.0                                             # log p about -1e-13: nearly all of its digits are in the rest
    z[3] *= 0.01
    z[4, 0] += 11.0
    _check_logprobs(z.to(dtype), _tokens(T, 3, V, V), min(V, 20))


@pytest.mark.parametrize("T, V", [(1, 131072), (2, 40000), (17, 9000), (300, 4000), (1500, 700), (4100, 130)])
@pytest.mark.parametrize("n_top", [0, 1, 32])
def test_logprobs_of_batches(T, V, n_top):
    z = torch.randn((T, V), generator=_gen(T)) * 4.0
    _check_logprobs(z.to(BF16) if n_top == 1 else z, _tokens(T, 2, V, T), n_top)


@pytest.mark.parametrize("V", [40, 3000, 70001])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_alternatives_of_hard_rows(V, dtype):
    """Equal entries (the lowest ids win), rows in rising and falling order, plateaus, the best at either end, signed zeros."""
    n = 32
    z = torch.zeros((9, V))
    z[1] = torch.arange(V) / 64.0 if dtype == FP32 else torch.arange(V) / 1000.0
    z[2] = -z[1]
    z[3] = (torch.arange(V) % 17).float()
    z[4, V - n:] = 1.0
    z[5, :n] = 1.0
    z[6, ::2] = -0.0
    z[7] = (torch.arange(V) // 100).float().clamp(max=30)
    z[8, V // 2] = 5.0
    _check_logprobs(z.to(dtype), _tokens(9, 1, V, V), n)


@pytest.mark.parametrize("V", [100, 5000, 140001])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_masked_rows(V, dtype):
    """Masks of -inf and of the type's lowest value, rows with one, a few and no entries left, NaN and infinity among them."""
    n = 12
    low = torch.finfo(dtype).min
    z = torch.randn((12, V), generator=_gen(V)) * 3
    keep = torch.randperm(V, generator=_gen(1))[:5]
    z[1] = -math.inf
    z[1, keep] = torch.tensor([1.0, 3.0, 3.0, -2.0, 0.0])         # fewer entries than alternatives: masked ones follow by id
    z[2] = -math.inf
    z[2, V - 1] = -1000.0                                           # one possible token
    z[3] = low
    z[3, keep] = torch.tensor([1.0, 3.0, 3.0, -2.0, 0.0])
    z[4] = low                                                      # uniform
    z[5, : V // 2] = -math.inf
    z[6, V // 2:] = -math.inf
    z[7] = -math.inf                                                # nothing left
    z[8, V // 2] = math.nan
    z[9, 3] = math.inf
    z[10] = math.nan
    z[11, V - 1], z[11, 0] = math.nan, -math.inf
    z = z.to(dtype)
    tokens = _tokens(12, 3, V, 3)
    tokens[:, 1], tokens[5, 2], tokens[7:, 2] = keep[1].item(), -1, V  # padding ids
    b = _check_logprobs(z, tokens, n, rows=list(range(7)))
    for t in range(7, 12):
        assert b.entropy[t].isnan() and b.conf[t].isnan() and b.top_logp[t].isnan().all() and b.token_logp[t, :2].isnan().all()
        assert b.token_logp[t, 2] == 0.0
        order = torch.sort(torch.where(z[t].isnan(), -math.inf, z[t].float()), descending=True, stable=True).indices[:n]
        assert torch.equal(b.top_idx[t].cpu().long(), order)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_logprobs_of_strided_rows_at_any_alignment(dtype):
    for V, ld, first in ((1000, 1003, 1), (20000, 20007, 3), (777, 777, 5)):
        mem = (torch.randn((first + 5 * ld,), generator=_gen(V)) * 3).to(dtype)
        at = mem.as_strided((5, V), (ld, 1), first)
        for t in range(5):                                          # what stands between the rows must not matter
            mem[first + t * ld + V: first + (t + 1) * ld] = math.nan
        _check_logprobs(at, _tokens(5, 64, V, 1), 8, view=mem.cuda().as_strided((5, V), (ld, 1), first))


def test_outputs_that_are_not_wanted():
    z = (torch.randn((3, 5000), generator=_gen(0)) * 3).cuda()
    full = mm.LogprobBuffers(3, 0, 4, 5000).run(z)
    b = mm.LogprobBuffers(3, 0, 4, 5000)
    b.entropy.fill_(9.0)
    mm.moe_token_logprobs(b.c[mm.MOE_FP32], z, None, None, None, None, b.top_idx, b.top_logp, b.ws, b.ws.numel())
    assert torch.equal(b.top_idx, full.top_idx) and torch.equal(b.top_logp, full.top_logp) and (b.entropy == 9.0).all()


def test_rows_do_not_depend_on_the_batch():
    """The same row alone, in a small and in a large batch: equal up to the order of additions, the alternatives exactly."""
    V = 30011
    z = (torch.randn((600, V), generator=_gen(0)) * 3)
    one, many = _check_logprobs(z[:1], _tokens(1, 1, V, 1), 9), _check_logprobs(z, _tokens(600, 1, V, 1), 9)
    assert torch.equal(one.top_idx[0], many.top_idx[0])
    assert torch.allclose(one.top_logp[0], many.top_logp[0], rtol=1e-5)


def test_rows_beyond_32_bit_offsets():
    """Logits whose last rows lie beyond 2^32 bytes and 2^31 elements."""
    T, V, ld = 3, 4000, 2 ** 22 - 1
    rows = 2 ** 31 // ld + T
    mem = torch.empty((rows * ld,), dtype=BF16, device="cuda")
    z = torch.randn((T, V), generator=_gen(0)).to(BF16)
    big = mem.as_strided((rows, V), (ld, 1))
    big.zero_()
    big[rows - T:] = z.cuda()
    b = mm.LogprobBuffers(rows, 0, 3, V).run(big)
    small = mm.LogprobBuffers(T, 0, 3, V).run(z.cuda())
    assert torch.equal(b.top_idx[rows - T:], small.top_idx)
    assert torch.allclose(b.entropy[rows - T:], small.entropy, rtol=1e-5) and (b.top_idx[:4] == torch.arange(3, device="cuda")).all()


@pytest.mark.parametrize("T, N", [(40, 70000), (300, 70000)])
def test_weights_and_outputs_beyond_32_bit_offsets(T, N):
    """Weights that reach beyond 2^32 bytes by their stride, outputs beyond 2^31 elements by theirs."""
    K, ldw, ldo = 96, 65536, 2 ** 22 - 1 if T == 300 else N
    mem = torch.empty((N * ldw,), dtype=torch.int8, device="cuda")
    w = mem.as_strided((N, K), (ldw, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    w.copy_(torch.randint(-128, 128, (N, K), generator=g, device="cuda").to(torch.int8))
    x, _, xs, _, _ = [t.cuda() for t in _operands(T, 1, K, seed=9)]
    ws = torch.rand((N,), generator=g, device="cuda") + 0.5
    outs = 2 ** 31 // ldo + 300 if T == 300 else T
    buf = torch.empty((outs * ldo,), dtype=BF16, device="cuda")
    out = buf.as_strided((outs, N), (ldo, 1))
    x = x.repeat((outs + T - 1) // T, 1)[:outs].contiguous()
    xs = xs.repeat((outs + T - 1) // T)[:outs].contiguous()
    mm.moe_matmul_int8(mm.int8_config(x[:, :K], w, out), x[:, :K], xs, w, ws, None, out)
    for rows in (slice(0, 5), slice(outs - 5, outs)):
        for cols in (slice(0, 100), slice(N - 100, N)):
            ref = (x[rows, :K].double().cpu() @ w[cols].double().cpu().t().contiguous()) * xs[rows].double().cpu()[:, None] * ws[cols].double().cpu()
            assert ((out[rows, cols].double().cpu() - ref).abs() <= _bound(ref, ref.abs(), BF16)).all()
