"""Plain implementations in 64 bits of the attention step's operators, on the CPU, and the error that fp32 arithmetic may make: what the tests of the kernels
compare with.  A cache is compared by the values that its stored rows stand for."""
from __future__ import annotations

import math

import torch

from paper_2510_12357_amd import binding as mm

BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
ULP = 2.0 ** -24                       # half a step of fp32, relative


def gen(seed):
    return torch.Generator().manual_seed(seed)


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def values(rows, scale=None):
    """fp64 values of a cache's rows."""
    x = rows.cpu().float().double()
    return x if scale is None else x * scale.cpu().double()[..., None]


# ---- rotary positions
def turned(x, pos, freq, layout, mscale=1.0, inverse=False):
    """x [tokens, heads, channels] -> fp64, by the definition."""
    x = x.cpu().double()
    half = freq.numel()
    t = pos.cpu().double()[:, None, None] * freq.cpu().double() * (-1.0 if inverse else 1.0)
    c, s = torch.cos(t) * mscale, torch.sin(t) * mscale
    out = x.clone()
    a_at, b_at = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    a, b = x[..., a_at], x[..., b_at]
    out[..., a_at], out[..., b_at] = a * c - b * s, b * c + a * s
    return out


def turn_error(x, freq, layout, mscale=1.0):
    """What fp32 may be off: sine and cosine by 2 half steps of 1 each (argument 1, series and sum 1), times m, product, sum: 1 each, 5 of |a| + |b| in all; 6."""
    x = x.cpu().double().abs()
    half = freq.numel()
    out = torch.zeros_like(x)
    a_at, b_at = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    out[..., a_at] = out[..., b_at] = (x[..., a_at] + x[..., b_at]) * abs(mscale) * 6 * ULP
    return out


def assert_near(got, want, error, dtype):
    """`error` in fp32 arithmetic, then rounded to dtype."""
    got = got.cpu().double()
    bound = error + (want.abs() + error) * half_step(dtype) * (1.0 if dtype != FP32 else 2.0) + 1e-40
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    off = torch.where(nan, 0.0, (got - want).abs() - bound)
    assert (off <= 0).all(), f"{int((off > 0).sum())} of {off.numel()} beyond the bound, worst {float(off.max()):.3g} at {int(off.argmax())}"


# ---- paged caches
class Paged:
    """A cache on the GPU whose rows are NaN but for those of the sequences, which lie on shuffled pages."""

    def __init__(self, lengths, page, heads, dim, dtype, seed, spare=3, far=0, layout="heads", extra_entries=2):
        g = gen(seed)
        counts = [-(-n // page) for n in lengths]
        total = sum(counts)
        self.n_pages = total + spare + far
        ids = (torch.randperm(total + spare, generator=g) + far).to(torch.int32)
        self.table = torch.full((len(lengths), max(counts + [0]) + extra_entries), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(counts):
            self.table[s, :n] = ids[at:at + n]
            at += n
        self.page, self.heads, self.dim, self.dtype, self.lengths = page, heads, dim, dtype, list(lengths)
        shape = (self.n_pages, heads, page, dim) if layout == "heads" else (self.n_pages, page, heads, dim)
        make = (lambda: torch.empty(shape, dtype=torch.uint8, device="cuda").fill_(0x7f).view(E4M3)) if dtype is E4M3 else \
            (lambda: torch.full(shape, math.nan, dtype=dtype, device="cuda"))
        self.k, self.v = ((t if layout == "heads" else t.permute(0, 2, 1, 3)) for t in (make(), make()))
        self.k_scale, self.v_scale = (torch.full((self.n_pages, heads, page), math.nan, device="cuda") if dtype is E4M3 else None for _ in range(2))
        self.cache = mm.KvCache(self.k, self.v, self.k_scale, self.v_scale)

    def slots(self, s, pos):
        pos = torch.as_tensor(pos)
        return self.table[s].long()[pos // self.page], pos % self.page

    def fill(self, seed, from_pos=None, k_gain=1.0):
        """Random rows at the positions that are seen (from from_pos[s] on) -> per sequence (k, v) in fp64 [positions, heads, channels]."""
        g, got = gen(seed), []
        for s, n in enumerate(self.lengths):
            lo = 0 if from_pos is None else from_pos[s]
            page, off = self.slots(s, torch.arange(lo, max(n, lo)))
            page, off = page.cuda(), off.cuda()
            pair = []
            for t, scale, gain in ((self.k, self.k_scale, k_gain), (self.v, self.v_scale, 1.0)):
                x = torch.randn((page.numel(), self.heads, self.dim), generator=g) * gain
                if self.dtype is E4M3:
                    a = x.abs().amax(dim=-1).clamp_min(1e-20) * (0.5 + torch.rand(x.shape[:2], generator=g))
                    codes, sc = (x / a[..., None] * 448.0).clamp(-448, 448).to(E4M3), (a / 448.0)
                    t.view(torch.uint8)[page, :, off] = codes.view(torch.uint8).cuda()
                    scale[page, :, off] = sc.cuda()
                    pair.append(values(codes, sc))
                else:
                    t[page, :, off] = x.to(self.dtype).cuda()
                    pair.append(values(x.to(self.dtype)))
            got.append(tuple(pair))
        return got


def attended(q, kv, scale, softcap=0.0):
    """One sequence: q [heads, channels], kv fp64 [positions, key heads, channels] of what is seen -> out, lse, and the error bounds of both.

    fp32: a score of D products is off by D steps of the sum of magnitudes (the matrix instructions may truncate: whole steps) and by 4 of itself (scale, units of log 2,
    maximum, cap); the exponential doubles nothing beyond that error and 4 steps of its own; sums over n positions by n steps of their magnitudes, as may the product with the values.
    Scales of 8-bit rows: a step more each."""
    k, v = kv
    H, D = q.shape
    n, Hk = k.shape[0], k.shape[1]
    if n == 0:
        z = torch.zeros((H, D), dtype=torch.float64)
        return z, torch.full((H,), -math.inf, dtype=torch.float64), z, torch.zeros(H, dtype=torch.float64)
    g = H // Hk
    q = q.cpu().double().view(Hk, g, D)
    raw = torch.matmul(k.permute(1, 0, 2).contiguous(), q.transpose(1, 2).contiguous()) * scale          # [key heads, positions, group]
    size = torch.matmul(k.abs().permute(1, 0, 2).contiguous(), q.abs().transpose(1, 2).contiguous()) * abs(scale)
    s = softcap * torch.tanh(raw / softcap) if softcap else raw
    ds = (2 * ULP) * ((D + 4) * size + 4 * s.abs() + (8 * softcap if softcap else 0.0))
    m = s.amax(dim=1, keepdim=True)
    ds = ds + 2 * ULP * m.abs()
    e = torch.exp(s - m)
    total = e.sum(dim=1, keepdim=True)
    p = (e / total).transpose(1, 2).contiguous()                                                         # [key heads, group, positions]
    dp = (e / total * (torch.expm1(ds) + 5 * 2 * ULP)).transpose(1, 2).contiguous()
    vv = v.permute(1, 0, 2).contiguous()
    out, mass = torch.matmul(p, vv), torch.matmul(p, vv.abs())
    dl = dp.sum(dim=2, keepdim=True) + n * 2 * ULP
    err = torch.matmul(dp, vv.abs()) + mass * (n + 4) * 2 * ULP + mass * dl
    lse = (m + torch.log(total)).reshape(H)
    return out.reshape(H, D), lse, err.reshape(H, D), (dl.reshape(H) + 4 * 2 * ULP * (1.0 + lse.abs() + m.reshape(H).abs()))
