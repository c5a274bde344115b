"""Attention over a paged cache where a workgroup's share is several pieces of 4096 positions: batches of long sequences, whose shares begin and end anywhere.  All sequences
of a batch have the same pages, so that a small cache is enough.  Bounds on sums of many positions let a lost one through, so most of these tests count them: with a scale of 0 each
has the same weight, and a result is the number of ones among the values over the number of positions."""
import math

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import BF16, E4M3, FP32, assert_near, attended, gen

pytestmark = pytest.mark.gpu
PAGE, HEADS, KV_HEADS, LONGEST, PIECE = 16, 16, 8, 40000, 4096
KINDS = [(BF16, BF16, 64), (BF16, E4M3, 64), (FP32, FP32, 64), (FP32, BF16, 64), (FP32, E4M3, 64), (BF16, BF16, 128), (BF16, E4M3, 128), (FP32, FP32, 128), (FP32, BF16, 256), (BF16, E4M3, 256)]


def _lengths(sequences, seed):
    """From a piece to all positions; at a piece's end, one behind it, nothing, and one."""
    n = torch.randint(PIECE, LONGEST + 1, (sequences,), generator=gen(seed))
    n[:7] = torch.tensor([LONGEST, 2 * PIECE, 2 * PIECE + 1, 0, 1, 3 * PIECE - 1, LONGEST - 1])
    return n[torch.randperm(sequences, generator=gen(seed + 1))].tolist()


class _Long:
    """A cache with all positions of one sequence, and a batch that sees it."""

    def __init__(self, cache, dim, sequences, window=0, seed=1):
        self.dim, self.window = dim, window
        self.lengths = _lengths(sequences, seed)
        order = torch.randperm(LONGEST // PAGE, generator=gen(seed))
        self.table = order.to(torch.int32)[None, :].repeat(sequences, 1)
        self.slot = order.repeat_interleave(PAGE) * PAGE + torch.arange(LONGEST) % PAGE         # of a position
        self.cache = mm.KvCache.empty(LONGEST // PAGE, PAGE, KV_HEADS, dim, cache)
        for t in (self.cache.k_scale, self.cache.v_scale):
            if t is not None:
                t.fill_(1.0)

    def put(self, t, rows):
        """Stores rows [positions, key heads, channels] -> what they are in the cache's type."""
        by_slot = torch.empty_like(rows)
        by_slot[self.slot] = rows
        rows = by_slot.view(-1, PAGE, KV_HEADS, self.dim).transpose(1, 2).to(t.dtype)
        if t.dtype is E4M3:
            t.view(torch.uint8).copy_(rows.contiguous().view(torch.uint8))
        else:
            t.copy_(rows)
        return rows.transpose(1, 2).reshape(LONGEST, KV_HEADS, self.dim).float()[self.slot]

    def seen(self, s):
        n = self.lengths[s]
        return (max(0, n - self.window) if self.window else 0), n

    def run(self, q, table=None, **kw):
        attn = mm.DecodeAttention(self.cache, HEADS, window=self.window, **kw)
        lse = torch.zeros(q.shape[:2], device="cuda")
        out = attn(q.cuda(), (self.table if table is None else table).cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda"), LONGEST, lse=lse)
        return attn, out.cpu().double(), lse.cpu().double()

    def share(self, attn):
        """Blocks of a workgroup's share, from the workspace that the call asked for: two segments' sums and statistics and four numbers a workgroup."""
        up = lambda n: -(-n // 256) * 256  # noqa: E731
        rows = 2 * min(16, HEADS // KV_HEADS)
        (w,) = [w for w in range(1, 4097) if up(w * rows * self.dim * 4) + up(w * rows * 8) + up(w * 16 + 4) == attn.ws.numel()]
        spans = [(lo // 64 * 64, n) for lo, n in map(self.seen, range(len(self.lengths)))]
        return sum(-(-(n - lo) // 64) + 4 for lo, n in spans if n) * KV_HEADS / w, w


@pytest.mark.parametrize("dtype, cache, dim", KINDS)
@pytest.mark.parametrize("sequences, window", [(60, 0), (60, 30000), (23, 0)])
def test_every_position_counts_once(dtype, cache, dim, sequences, window):
    """fp32 results: every position has ones in its own random channels.  bf16 ones, which have 8 bits: the first and the last position of every block, in turn over the
    channels, at most 20 to a channel.  Weights and sums of ones are exact; a quotient, its rounding and bf16's are less than 2^-8 of the result, 0.1 of 20 ones, and 2^-22, 0.01 of 40000 ones."""
    b = _Long(cache, dim, sequences, window, seed=dim)
    ones = torch.zeros((LONGEST, KV_HEADS, dim))
    if dtype is FP32:
        ones = (torch.rand(ones.shape, generator=gen(5)) < 0.5).float()
    else:
        at = torch.cat([torch.arange(0, LONGEST, 64), torch.arange(63, LONGEST, 64)]).sort().values
        for h in range(KV_HEADS):
            ones[at, h, (torch.arange(at.numel()) + 7 * h) % dim] = 1.0
    b.put(b.cache.k, torch.randint(-3, 4, ones.shape, generator=gen(6)).float())
    b.put(b.cache.v, ones)
    q = torch.randn((sequences, HEADS, dim), generator=gen(7)).to(dtype)
    attn, out, lse = b.run(q, scale=0.0)
    share, workgroups = b.share(attn)
    assert workgroups < sequences * KV_HEADS * (LONGEST // 512) and (share > 2 * 64 if sequences == 60 and window == 0 else share > 32), (share, workgroups)
    upto = torch.cat([torch.zeros((1, KV_HEADS, dim), dtype=torch.float64), ones.double().cumsum(0)])
    for s in range(sequences):
        lo, n = b.seen(s)
        if n == 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            continue
        want = (upto[n] - upto[lo]).repeat_interleave(HEADS // KV_HEADS, 0)
        assert (out[s] * (n - lo) - want).abs().max() < 0.25, (s, lo, n)
        # the logarithm of a whole number, below 16: two steps of 2^-20; one position changes it by 1 / n > 2^-16
        assert (lse[s] - math.log(n - lo)).abs().max() <= 2.0 ** -19, (s, lo, n)


@pytest.mark.parametrize("dtype, cache, dim", KINDS)
def test_scores_that_jump_at_pieces(dtype, cache, dim):
    """Positions beside the borders of pieces have most of the weight, in rising order, so that sums are rescaled from piece to piece; the definition in 64 bits of some sequences."""
    b = _Long(cache, dim, 60, seed=dim + 1)
    k = torch.randint(-8, 9, (LONGEST, KV_HEADS, dim), generator=gen(1)).float() / 8
    at = torch.cat([torch.arange(0, LONGEST, PIECE // 2) + i for i in (-65, -64, -1, 0, 1, 63, 64)]).sort().values
    at = at[(at >= 0) & (at < LONGEST)]
    k[:, :, 0] = -1.0
    k[at, :, 0] = 8.0 + (torch.arange(at.numel()) // 14 * 0.5).clamp(max=7.0)[:, None]
    v = torch.randint(-8, 9, k.shape, generator=gen(2)).float() / 8
    k, v = b.put(b.cache.k, k), b.put(b.cache.v, v)
    q = torch.randn((60, HEADS, dim), generator=gen(3)) * 0.25
    q[:, :, 0] = 2.0
    q = q.to(dtype)
    attn, out, lse = b.run(q, scale=0.5)
    assert b.share(attn)[0] > 2 * 64
    for s in sorted({b.lengths.index(n) for n in (LONGEST, 2 * PIECE, 2 * PIECE + 1, 1, 3 * PIECE - 1)} | {20, 40}):
        n = b.lengths[s]
        want, want_lse, err, lse_err = attended(q[s], (k[:n].double(), v[:n].double()), 0.5)
        assert_near(out[s].to(dtype), want, err, dtype)
        assert ((lse[s] - want_lse).abs() <= lse_err).all()


@pytest.mark.parametrize("dtype, cache, dim", KINDS[:5])
def test_a_page_that_does_not_exist_in_any_piece(dtype, cache, dim):
    """In the first, a middle and the last piece of a sequence: NaN there, and nowhere else."""
    b = _Long(cache, dim, 60, seed=3)
    for t, seed in ((b.cache.k, 1), (b.cache.v, 2)):
        b.put(t, torch.randint(-8, 9, (LONGEST, KV_HEADS, dim), generator=gen(seed)).float() / 8)
    q = torch.randn((60, HEADS, dim), generator=gen(3)).to(dtype)
    attn, out, lse = b.run(q)
    assert b.share(attn)[0] > 2 * 64 and torch.isfinite(out).all()
    table, bad = b.table.clone(), []
    for s in range(0, 60, 3):
        n = b.lengths[s]
        if n < 2 * PIECE:
            continue
        at = (0, n // 2, n - 1, PIECE, PIECE - 1)[s // 3 % 5]
        table[s, at // PAGE] = (-1, b.cache.n_pages, 2 ** 31 - 1)[s // 3 % 3]
        bad.append(s)
    _, spoiled, spoiled_lse = b.run(q, table)
    assert len(bad) > 10
    for s in range(60):
        if s in bad:
            assert spoiled[s].isnan().all() and spoiled_lse[s].isnan().all(), s
        else:
            assert torch.equal(spoiled[s], out[s]) and torch.equal(spoiled_lse[s], lse[s]), s
