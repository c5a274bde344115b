"""Rotary positions and appends to a paged cache against the definitions in 64 bits."""
import math

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import BF16, E4M3, FP32, ULP, Paged, assert_near, gen, turn_error, turned, values

pytestmark = pytest.mark.gpu


def _rotary(rotary, layout, mscale=1.0, factor=1.0):
    return mm.Rotary.scaled(rotary, layout=layout, mscale=mscale, factor=factor, trained=4096 if factor != 1.0 else 0)


def _positions(T, far, seed):
    pos = torch.randint(0, far, (T,), generator=gen(seed))
    pos[: T // 4] = torch.arange(T // 4)
    pos[-1] = far - 1
    return pos.to(torch.int32)


@pytest.mark.parametrize("T, heads, dim, rotary, far", [
    (1, 1, 2, 2, 1), (1, 32, 128, 128, 4096), (3, 5, 64, 64, 100), (7, 3, 80, 48, 1 << 20), (65, 2, 256, 256, 1 << 31), (33, 4, 96, 20, 5000), (129, 1, 250, 18, 9),
    (5, 9, 66, 0 + 2, 777), (257, 40, 128, 64, 131072), (2100, 7, 36, 36, 50000), (2, 70, 256, 2, 3),
])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rotation(T, heads, dim, rotary, far, layout, dtype):
    rot = _rotary(rotary, layout, mscale=1.1 if heads % 2 else 1.0, factor=4.0 if T % 2 else 1.0)
    x = (torch.randn((T, heads, dim), generator=gen(1)) * 3).to(dtype)
    pos = _positions(T, far, 2)
    out = rot(x.cuda(), pos.cuda())
    want = turned(x, pos, rot.freq, layout, rot.mscale)
    assert_near(out, want, turn_error(x, rot.freq, layout, rot.mscale), dtype)
    assert torch.equal(out.cpu()[..., rotary:], x[..., rotary:])
    # in place, and turned back
    again = x.cuda()
    rot(again, pos.cuda(), out=again)
    assert torch.equal(again, out)
    back = rot(x.cuda(), pos.cuda(), inverse=True)
    assert_near(back, turned(x, pos, rot.freq, layout, rot.mscale, inverse=True), turn_error(x, rot.freq, layout, rot.mscale), dtype)


def test_gradient_is_the_rotation_back():
    """<g, turn(x)> changes with x by turn_back(g): against differences of the kernel's own values in fp32."""
    rot = _rotary(16, "half", mscale=1.25)
    x, g = torch.randn((6, 2, 24), generator=gen(1)), torch.randn((6, 2, 24), generator=gen(2))
    pos = _positions(6, 300, 3).cuda()
    grad = rot(g.cuda(), pos, inverse=True).cpu().double()
    for at in [(0, 0, 0), (1, 1, 7), (2, 0, 8), (3, 1, 15), (5, 0, 16), (5, 1, 23)]:
        hi, lo = x.clone(), x.clone()
        hi[at] += 1.0
        lo[at] -= 1.0
        d = (rot(hi.cuda(), pos).cpu().double() - rot(lo.cuda(), pos).cpu().double())
        size = ((hi.abs() + lo.abs()).double() * g.abs().double()).sum()
        # the map is linear: a difference over 2 has no error but the arithmetic's
        assert abs(float((g.double() * d).sum() / 2 - grad[at])) <= float(size) * 1.25 * 16 * ULP + 16 * ULP * float(g.abs().max())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_strides_and_negative_positions(layout):
    rot = _rotary(32, layout)
    rows = torch.randn((9, 5, 71), generator=gen(1)).to(BF16).cuda()
    x = rows[1:8:2, 1:4, 3:67]                                # odd strides and an odd start
    pos = torch.tensor([-5, 0, -(1 << 31), 2 ** 31 - 1], dtype=torch.int32)
    want, err = turned(x, pos, rot.freq, layout), turn_error(x, rot.freq, layout)
    assert_near(rot(x, pos.cuda()), want, err, BF16)
    heads_first = x.transpose(0, 1).contiguous().transpose(0, 1)          # heads outside
    assert_near(rot(heads_first, pos.cuda()), want, err, BF16)
    into = torch.full((4, 7, 70), 5.0, dtype=BF16, device="cuda")
    rot(x, pos.cuda(), out=into[:, 2:5, 1:65])
    assert_near(into[:, 2:5, 1:65], want, err, BF16)
    into[:, 2:5, 1:65] = 5.0
    assert (into == 5.0).all()


def test_values_that_are_none_stay_in_their_pair():
    rot = _rotary(16, "half")
    x = torch.randn((1, 1, 32), generator=gen(1)).cuda()
    x[0, 0, 3], x[0, 0, 20], x[0, 0, 21] = math.nan, math.inf, math.nan
    out = rot(x, torch.tensor([7], dtype=torch.int32, device="cuda")).cpu()[0, 0]
    assert torch.isnan(out).nonzero().flatten().tolist() == [3, 11, 21] and out[20] == math.inf


def test_other_frequencies():
    """Any list of them; by parts, slow ones are divided by the factor, fast ones are kept."""
    rot = mm.Rotary.scaled(64, factor=8.0, trained=4096, slow=1.0, fast=4.0)
    plain = mm.Rotary.scaled(64)
    f, p = rot.freq.cpu(), plain.freq.cpu()
    turns = 4096 * p / (2 * math.pi)
    assert torch.equal(f[turns >= 4], p[turns >= 4]) and torch.allclose(f[turns <= 1], p[turns <= 1] / 8, rtol=1e-15) and (f[:-1] > f[1:]).all()
    assert torch.allclose(mm.Rotary.scaled(64, factor=8.0).freq.cpu(), p / 8, rtol=1e-15)
    freq = torch.tensor([0.0, 1e-12, 3.0], dtype=torch.float64, device="cuda")
    x, pos = torch.randn((4, 1, 6), generator=gen(1)), torch.tensor([0, 1, 10 ** 9, 2 ** 31 - 1], dtype=torch.int32)
    own = mm.Rotary(freq, "interleaved", 0.5)
    assert_near(own(x.cuda(), pos.cuda()), turned(x, pos, freq, "interleaved", 0.5), turn_error(x, freq, "interleaved", 0.5), FP32)


def test_no_tokens_and_refusals():
    rot = _rotary(16, "half")
    none = torch.empty((0, 4, 32), device="cuda")
    assert rot(none, torch.empty((0,), dtype=torch.int32, device="cuda")).shape == none.shape
    x, pos = torch.ones((2, 3, 32), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: rot(x, pos.long()), lambda: rot(x, pos[:1]), lambda: rot(x.cpu(), pos), lambda: rot(x, pos.cpu()), lambda: rot(x[0], pos),
                lambda: rot(x, pos, out=x.to(BF16)), lambda: rot(x, pos, out=x[:, :2]), lambda: rot(x.expand(2, 3, 32)[:1].expand(2, 3, 32), pos),
                lambda: rot(x.transpose(1, 2), pos), lambda: mm.Rotary(rot.freq.float()), lambda: mm.Rotary(rot.freq.cpu()), lambda: mm.Rotary(rot.freq, "other"),
                lambda: mm.Rotary.scaled(7), lambda: mm.Rotary.scaled(8, factor=0.0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mm.MoeError):
        rot(torch.ones((2, 3, 8), device="cuda"), pos)       # fewer channels than turn
    with pytest.raises(KeyError):
        rot(x.half(), pos)


# ------------------------------------------------------------------------------------ appends
def _check_rows(p, name, s, pos, want, err):
    """The stored rows of sequence s at `pos` against fp64 rows [positions, heads, channels] that are exact to err."""
    t, scale = getattr(p, name), getattr(p, name + "_scale")
    page, off = p.slots(s, pos)
    got = t.view(torch.uint8).cpu().view(t.dtype) if t.dtype is E4M3 and t.is_contiguous() else t.cpu()
    rows = got.view(torch.uint8)[page, :, off].view(t.dtype) if t.dtype is E4M3 else got[page, :, off]
    if scale is None:
        assert_near(rows, want, err, t.dtype)
        return
    scales = scale.cpu()[page, :, off]
    a = want.abs().amax(dim=-1)
    # two roundings of the quotient, and the row's error
    assert ((scales.double() - a / 448).abs() <= (a * 2 * ULP + err.amax(dim=-1)) / 448 + 1e-44).all()
    # nearest codes: half a step of e4m3 (of the smallest numbers 2^-10), the quotient's own roundings in front of it
    exact = torch.where(a[..., None] > 0, want / (a / 448)[..., None], 0.0)
    slack = torch.where(a[..., None] > 0, err / (a / 448)[..., None], 0.0) + exact.abs() * 8 * ULP
    step = torch.clamp(exact.abs() * 2.0 ** -4, min=2.0 ** -10)
    assert ((values(rows) - exact).abs() <= step + 2 * slack).all()


@pytest.mark.parametrize("cache", [BF16, FP32, E4M3])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("dim, rotary, layout, page, heads, kv_heads", [
    (128, 128, "half", 16, 8, 2), (64, 64, "interleaved", 4, 3, 3), (80, 48, "half", 64, 5, 1), (96, 20, "interleaved", 32, 4, 2), (16, 2, "half", 8, 1, 1),
    (256, 256, "half", 16, 2, 2), (256, 18, "interleaved", 256, 2, 1), (48, 0, "half", 16, 2, 2),
])
def test_append_of_ragged_chunks(cache, dtype, dim, rotary, layout, page, heads, kv_heads):
    """Chunks of three sequences in any order with padding among them; everything else in the cache is as it was."""
    before, new = [0, 5, 37, 0], [1, 21, 40, 0]
    p = Paged([b + n for b, n in zip(before, new)], page, kv_heads, dim, cache, seed=3)
    T = sum(new) + 3
    g = gen(dim + page)
    rows = torch.randn((T, heads + 2 * kv_heads, dim), generator=g).to(dtype)
    rows[5, :, :] = 0.0
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:]
    where = [(s, b + i) for s, (b, n) in enumerate(zip(before, new)) for i in range(n)] + [(0, -1), (2, -7), (1, -(1 << 31))]
    order = torch.randperm(T, generator=g).tolist()
    where = [where[i] for i in order]
    seq, pos = (torch.tensor([w[i] for w in where], dtype=torch.int32) for i in (0, 1))
    rot = _rotary(rotary, layout, mscale=1.2) if rotary else None
    old = [None if t is None else t.clone() for t in (p.k, p.v, p.k_scale, p.v_scale)]
    d = rows.cuda()
    q_out = p.cache.append(d[:, heads:heads + kv_heads], d[:, heads + kv_heads:], pos.cuda(), p.table.cuda(), seq=seq.cuda(), rotary=rot, q=d[:, :heads])
    turn = (lambda x: (turned(x, pos, rot.freq, layout, 1.2), turn_error(x, rot.freq, layout, 1.2))) if rot else (lambda x: (x.double(), torch.zeros_like(x, dtype=torch.float64)))
    assert_near(q_out, *turn(q), dtype)
    want_k, err_k = turn(k)
    for s in range(3):
        t = [i for i in range(T) if where[i][0] == s and where[i][1] >= 0]
        at = [where[i][1] for i in t]
        _check_rows(p, "k", s, at, want_k[t], err_k[t])
        _check_rows(p, "v", s, at, v.double()[t], torch.zeros_like(want_k[t]))
    # nothing else was written
    hit = torch.zeros((p.n_pages, page), dtype=torch.bool)
    for s, o in where:
        if o >= 0:
            hit[p.table[s, o // page], o % page] = True
    hit = hit[:, None, :].expand(-1, kv_heads, -1).cuda()
    for now, was in zip((p.k, p.v, p.k_scale, p.v_scale), old):
        if now is not None:
            b = lambda t: t.contiguous().view(torch.uint8).view(p.n_pages, kv_heads, page, -1)  # noqa: E731
            assert torch.equal(b(now)[~hit], b(was)[~hit])


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_pages_that_do_not_exist_are_not_written(cache):
    p = Paged([20, 20, 20], 16, 2, 32, cache, seed=1, extra_entries=0)
    table = p.table.clone()
    table[0, 1], table[1, 1] = p.n_pages, -1
    old = p.k.view(torch.uint8).clone() if cache is E4M3 else p.k.clone()
    k = torch.ones((6, 2, 32), dtype=BF16, device="cuda")
    pos = torch.tensor([17, 18, 32, 2 ** 31 - 1, 3, 4], dtype=torch.int32, device="cuda")
    seq = torch.tensor([0, 1, 2, 2, 3, -1], dtype=torch.int32, device="cuda")
    q = torch.randn((6, 2, 32), generator=gen(2)).to(BF16).cuda()
    out = p.cache.append(k, k.clone(), pos, table.cuda(), seq=seq, rotary=_rotary(32, "half"), q=q)
    now = p.k.view(torch.uint8) if cache is E4M3 else p.k
    assert torch.equal(now.contiguous().view(torch.uint8), old.contiguous().view(torch.uint8))
    assert torch.isfinite(out).all()


def test_rows_of_eight_bits_that_hold_no_numbers():
    p = Paged([4], 4, 1, 64, E4M3, seed=1)
    k = torch.randn((4, 1, 64), generator=gen(1))
    k[0, 0, 3], k[1, 0, 60], k[2] = math.nan, -math.inf, 0.0
    k[3] *= 1e-38
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    p.cache.append(k.cuda(), k.cuda().clone(), pos, p.table.cuda(), seq=torch.zeros(4, dtype=torch.int32, device="cuda"))
    page = int(p.table[0, 0])
    for t, scale in ((p.k, p.k_scale), (p.v, p.v_scale)):
        scale = scale.cpu()[page, 0]
        assert torch.isnan(scale[:2]).all() and scale[2] == 0 and 0 < scale[3] < 1e-38
        assert (t.view(torch.uint8).cpu()[page, 0, :3] & 0x7f == 0).all() and t.float().cpu()[page, 0, 3].abs().max() == 448


@pytest.mark.parametrize("layout", ["heads", "positions"])
def test_one_token_each_in_both_orders_of_the_cache(layout):
    """Decode: token t is of sequence t; queries in place; a table cut out of a wider one."""
    lengths = [1, 16, 17, 33, 100]
    p = Paged(lengths, 16, 4, 64, BF16, seed=2, layout=layout, extra_entries=3)
    wide = torch.full((5, p.table.shape[1] + 4), 99999, dtype=torch.int32)
    wide[:, :p.table.shape[1]] = p.table
    k, v, q = (torch.randn((5, h, 64), generator=gen(h)).to(BF16) for h in (4, 4, 8))
    v = v.flip(0)
    pos = torch.tensor(lengths, dtype=torch.int32) - 1
    rot = _rotary(64, "half")
    dq = q.cuda()
    assert p.cache.append(k.cuda(), v.cuda(), pos.cuda(), wide.cuda()[:, :p.table.shape[1]], rotary=rot, q=dq, q_out=dq) is dq
    assert_near(dq, turned(q, pos, rot.freq, "half"), turn_error(q, rot.freq, "half"), BF16)
    for s, n in enumerate(lengths):
        _check_rows(p, "k", s, [n - 1], turned(k, pos, rot.freq, "half")[s:s + 1], turn_error(k, rot.freq, "half")[s:s + 1])
        _check_rows(p, "v", s, [n - 1], v.double()[s:s + 1], torch.zeros((1, 4, 64), dtype=torch.float64))


def test_append_refusals():
    p = Paged([20], 16, 2, 32, BF16, seed=1)
    k, pos, table = torch.ones((2, 2, 32), dtype=BF16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), p.table.cuda()
    a = p.cache.append
    assert a(k, k, pos, table, seq=pos) is None
    assert a(k[:0], k[:0], pos[:0], table, q=k[:0]).shape == (0, 2, 32)
    for bad in (lambda: a(k[:, :1], k[:, :1], pos, table), lambda: a(k, k.float(), pos, table), lambda: a(k, k[:1], pos, table), lambda: a(k.cpu(), k, pos, table),
                lambda: a(k, k, pos[:1], table), lambda: a(k, k, pos.long(), table), lambda: a(k, k, pos, table.long()), lambda: a(k, k, pos, table[0]),
                lambda: a(k, k, pos, table, seq=pos[:1]), lambda: a(k, k, pos, table, seq=pos.cpu()), lambda: a(k, k, pos, table, q_out=k),
                lambda: a(k, k, pos, table, q=k.float()), lambda: a(k, k, pos, table, q=k[:1]), lambda: a(k, k, pos, table, q=k[..., :16]),
                lambda: a(k, k, pos, table, q=k, q_out=k.cpu()), lambda: a(k[:1].expand(2, 2, 32), k, pos, table),
                lambda: a(k, k, pos, table[:1].expand(3, table.shape[1]))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mm.MoeError):
        a(k, k, pos, table, rotary=_rotary(64, "half"))      # more channels than there are
    f8 = torch.zeros((3, 2, 16, 32), dtype=E4M3, device="cuda")
    for bad in (lambda: mm.KvCache(f8, f8.clone()), lambda: mm.KvCache(p.k, p.v.float()), lambda: mm.KvCache(p.k.cpu(), p.v), lambda: mm.KvCache(p.k, p.v[:1]),
                lambda: mm.KvCache(p.k, p.v, torch.ones(p.k.shape[:3], device="cuda"), torch.ones(p.k.shape[:3], device="cuda")),
                lambda: mm.KvCache(p.k.transpose(2, 3), p.v.transpose(2, 3)), lambda: mm.KvCache(p.k.half(), p.v.half()),
                lambda: mm.KvCache(p.k[:1].expand(4, 2, 16, 32), p.v[:1].expand(4, 2, 16, 32))):
        with pytest.raises(ValueError):
            bad()
