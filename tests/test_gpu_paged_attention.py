"""Attention of one new token per sequence over a paged cache against the definition in 64 bits.  What is not seen is NaN in every cache here."""
import math

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import BF16, E4M3, FP32, Paged, assert_near, attended, gen

pytestmark = pytest.mark.gpu


def _check(p, kv, q, out, lse=None, scale=None, window=0, softcap=0.0, lengths=None, only=None):
    scale = 1.0 / math.sqrt(p.dim) if scale is None else scale
    for s, n in enumerate(p.lengths if lengths is None else lengths):
        if only is not None and s not in only:
            continue
        lo = max(0, n - window) if window else 0
        want, want_lse, err, lse_err = attended(q[s], (kv[s][0][lo:n], kv[s][1][lo:n]), scale, softcap)
        assert_near(out[s], want, err, out.dtype)
        if lse is not None:
            got = lse[s].cpu().double()
            assert ((got == want_lse) | ((got - want_lse).abs() <= lse_err)).all(), (s, n)


def _run(lengths, page, heads, kv_heads, dim, dtype, cache, seed=0, max_len=None, window=0, softcap=0.0, scale=None, gain=1.0, layout="heads", far=0):
    p = Paged(lengths, page, kv_heads, dim, cache, seed=seed, layout=layout, far=far)
    kv = p.fill(seed + 1, [max(0, n - window) if window else 0 for n in lengths])
    if window:                                               # from the first position on, so that rows are found by position
        kv = [tuple(torch.cat([torch.zeros((max(0, n - window),) + t.shape[1:], dtype=torch.float64), t]) for t in pair) for n, pair in zip(lengths, kv)]
    q = (torch.randn((len(lengths), heads, dim), generator=gen(seed + 2)) * gain).to(dtype)
    attn = mm.DecodeAttention(p.cache, heads, scale=scale, window=window, softcap=softcap)
    lse = torch.full((len(lengths), heads), math.nan, device="cuda")
    most = max(lengths + [0]) if max_len is None else max_len
    out = attn(q.cuda(), p.table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), most, lse=lse)
    _check(p, kv, q, out, lse, scale, window, softcap)
    return p, kv, q, attn, out, lse


EDGES = [0, 1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cache", [BF16, FP32, E4M3])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 144, 192, 256])
def test_every_width_at_every_edge_of_a_block(dtype, cache, dim):
    _run(EDGES, 16, 4, 2, dim, dtype, cache, seed=dim)


@pytest.mark.parametrize("group", [1, 2, 5, 15, 16, 17, 32, 33, 71])
@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_groups_of_heads(group, cache):
    _run([1, 40, 0, 300], 8, group * 2, 2, 64, BF16, cache, seed=group)
    _run([77, 130], 32, group, 1, 128, FP32, cache, seed=group)


@pytest.mark.parametrize("page", [4, 8, 32, 64, 128, 1024, 1 << 14])
@pytest.mark.parametrize("layout", ["heads", "positions"])
def test_pages_that_end_inside_and_outside_of_blocks(page, layout):
    _run([1, page, page + 1, 2 * page - 1 if page < 2000 else 900, 333], page, 4, 2, 128, BF16, BF16, seed=page, layout=layout)
    _run([700, 3, 1100], page, 4, 2, 64, BF16, E4M3, seed=page)


@pytest.mark.parametrize("cache, dim", [(BF16, 128), (BF16, 64), (E4M3, 128), (FP32, 64), (E4M3, 256), (BF16, 80)])
@pytest.mark.parametrize("lengths, max_len", [([5000], None), ([1, 0, 4096, 4097, 4999, 511, 512, 513], 6000), ([9000, 30], 20000), ([3], 100000)])
def test_parts_of_long_sequences(cache, dim, lengths, max_len):
    _run(lengths, 16, 8, 2, dim, BF16, cache, seed=dim, max_len=max_len)


@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP32, FP32), (BF16, E4M3)])
@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100, 128, 1000, 5000])
def test_windows(window, dtype, cache):
    """Pages in front of the window hold NaN, and their numbers need not exist."""
    lengths = [0, 1, window, window + 1, 64, 65, 300, 1500, 4100]
    p, kv, q, attn, out, _ = _run(lengths, 16, 4, 2, 64, dtype, cache, seed=window, window=window)
    table = p.table.clone()
    for s, n in enumerate(lengths):
        table[s, :max(0, n - window) // 16] = -1 if s % 2 else 2 ** 31 - 1
    again = attn(q.cuda(), table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max(lengths))
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype, cache", [(BF16, BF16), (FP32, FP32), (FP32, E4M3)])
@pytest.mark.parametrize("softcap, scale, gain", [(30.0, None, 4.0), (2.0, 0.3, 10.0), (0.0, 1.0, 8.0), (0.0, -0.4, 3.0), (0.0, 0.0, 1.0)])
def test_scales_and_caps(dtype, cache, softcap, scale, gain):
    _run([1, 30, 333, 2500], 16, 6, 3, 64, dtype, cache, seed=3, softcap=softcap, scale=scale, gain=gain)


def test_a_maximum_that_grows_block_by_block():
    """Scores that rise and fall over the sequence by hundreds, so that sums are rescaled often and early ones vanish."""
    for order in ("up", "down", "late"):
        p = Paged([3000], 16, 1, 64, FP32, seed=1)
        (k, v), = p.fill(2)
        ramp = torch.linspace(-40, 40, 3000, dtype=torch.float64) if order != "late" else torch.where(torch.arange(3000) == 2999, 80.0, -10.0).double()
        k = (torch.ones((3000, 1, 64)).double() * (ramp if order != "down" else ramp.flip(0))[:, None, None]).float().double()
        page, off = p.slots(0, torch.arange(3000))
        p.k[page.cuda(), :, off.cuda()] = k.float().cuda()
        q = torch.ones((1, 3, 64)) + torch.randn((1, 3, 64), generator=gen(3)) * 0.1
        out = mm.DecodeAttention(p.cache, 3, scale=0.25)(q.cuda(), p.table.cuda(), torch.tensor([3000], dtype=torch.int32, device="cuda"), 3000)
        _check(p, [(k, v)], q, out, scale=0.25)


def test_strides_of_queries_outputs_and_tables():
    lengths = [40, 1, 333]
    p = Paged(lengths, 16, 2, 64, BF16, seed=1)
    kv = p.fill(2)
    rows = torch.randn((3, 9, 71), generator=gen(3)).to(BF16).cuda()
    q = rows[:, 2:8, 5:69]
    wide = torch.full((6, p.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[::2, :p.table.shape[1]] = p.table.cuda()
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    attn = mm.DecodeAttention(p.cache, 6)
    into = torch.full((3, 8, 66), 7.0, dtype=BF16, device="cuda")
    attn(q, wide[::2, :p.table.shape[1]], n, 333, out=into[:, 1:7, 1:65])
    _check(p, kv, q.cpu(), into[:, 1:7, 1:65])
    into[:, 1:7, 1:65] = 7.0
    assert (into == 7.0).all()
    heads_first = q.transpose(0, 1).contiguous().transpose(0, 1)
    _check(p, kv, q.cpu(), attn(heads_first, wide[::2, :p.table.shape[1]], n, 333))
    assert (attn(q[:0], wide[:0], n[:0], 333).shape == (0, 6, 64))


@pytest.mark.parametrize("cache", [BF16, E4M3])
@pytest.mark.parametrize("max_len", [700, 7000])
def test_what_is_wrong_with_one_sequence_spoils_that_one(cache, max_len):
    """Lengths and pages that do not exist: NaN in that sequence, the others as ever; with one part and with several."""
    lengths = [100, 0, 500, 30, 600, 64]
    p = Paged(lengths, 16, 2, 64, cache, seed=1, extra_entries=0)
    kv = p.fill(2)
    q = torch.randn((6, 4, 64), generator=gen(3)).to(BF16)
    attn = mm.DecodeAttention(p.cache, 4)
    for what in ("negative", "above", "table", "page", "pages", "far"):
        table, n, most = p.table.clone(), list(lengths), max_len
        if what == "negative":
            n[2] = -1
        elif what == "above":
            n[2], most = 600, 600
            n[2] = 601
        elif what == "table":
            n[2], most = p.table.shape[1] * 16 + 1, 100000
        elif what == "page":
            table[2, 20] = -1
        elif what == "pages":
            table[2, :] = p.n_pages
        else:
            table[2, 31] = 2 ** 31 - 1
        lse = torch.zeros((6, 4), device="cuda")
        out = attn(q.cuda(), table.cuda(), torch.tensor(n, dtype=torch.int32, device="cuda"), most, lse=lse)
        assert torch.isnan(out[2]).all() and torch.isnan(lse[2]).all(), what
        _check(p, kv, q, out, lse, only={0, 1, 3, 4, 5})


def test_values_that_are_no_numbers_show():
    """A NaN or an infinity in what is seen gives NaN in its channels, in a key in all."""
    for spot in (0, 100, 2047):
        for bad in (math.nan, math.inf):
            p = Paged([2048, 2048], 16, 2, 64, BF16, seed=1)
            kv = p.fill(2)
            page, off = p.slots(0, [spot])
            q = torch.randn((2, 4, 64), generator=gen(3)).to(BF16)
            n = torch.full((2,), 2048, dtype=torch.int32, device="cuda")
            attn = mm.DecodeAttention(p.cache, 4)
            p.v[page.cuda(), 1, off.cuda(), 5] = bad
            out = attn(q.cuda(), p.table.cuda(), n, 2048).cpu()
            assert not torch.isfinite(out[0, 2:, 5]).any()
            assert torch.isfinite(out[0, :2]).all() and torch.isfinite(out[0, :, :5]).all() and torch.isfinite(out[0, :, 6:]).all()
            _check(p, kv, q, out, only={1})
            p.k[page.cuda(), 0, off.cuda(), 9] = math.nan
            out = attn(q.cuda(), p.table.cuda(), n, 2048).cpu()
            assert torch.isnan(out[0, :2]).all()
            _check(p, kv, q, out, only={1})


@pytest.mark.parametrize("max_len", [40, 4000])
def test_scores_that_are_all_minus_infinity(max_len):
    """As an empty sequence: zeros, lse -inf; a single finite score among them has all the weight."""
    p = Paged([40, 40], 16, 1, 64, FP32, seed=1)
    kv = p.fill(2)
    q = torch.ones((2, 2, 64)) * 1e30
    page, off = p.slots(0, torch.arange(40))
    p.k[page.cuda(), :, off.cuda()] = -1e30
    page, off = p.slots(1, torch.arange(40))
    p.k[page.cuda(), :, off.cuda()] = -1e30
    p.k[page[33], :, off[33]] = 0.0
    lse = torch.zeros((2, 2), device="cuda")
    out = mm.DecodeAttention(p.cache, 2)(q.cuda(), p.table.cuda(), torch.tensor([40, 40], dtype=torch.int32, device="cuda"), max_len, lse=lse)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert torch.equal(out[1].cpu().double(), kv[1][1][33].expand(2, 64)) and (lse[1] == 0).all()


def test_the_same_call_has_the_same_bits_and_shares_pages():
    """Again; and sequences that have the same pages, as the definition has them (which parts a row has goes by the whole batch)."""
    p, kv, q, attn, out, lse = _run([3000, 50, 3000], 16, 8, 2, 128, BF16, BF16, seed=5)
    table, n = p.table.cuda(), torch.tensor([3000, 50, 3000], dtype=torch.int32, device="cuda")
    for _ in range(3):
        assert torch.equal(attn(q.cuda(), table, n, 3000), out)
    pick = torch.tensor([2, 2, 0], device="cuda")
    again = attn(q.cuda()[pick], table[pick], n[pick], 3000)
    for i, s in enumerate([2, 2, 0]):
        want, _, err, _ = attended(q[s], kv[s], 1.0 / math.sqrt(128))
        assert_near(again[i], want, err, BF16)


@pytest.mark.parametrize("lengths, max_len", [([700, 3, 1900], None), ([5000, 9000], None), ([300] * 70, None)])
def test_parts_joined_by_a_second_launch_and_results_in_place_of_the_queries(lengths, max_len):
    """Without counters the C call joins parts in a launch of its own, to the same values; and out may be q."""
    p, kv, q, attn, out, lse = _run(lengths, 16, 8, 2, 64, BF16, BF16, seed=7)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    c = mm.moe_attention_config()
    c.B, c.heads, c.dtype, c.max_len, c.table_len, c.scale = len(lengths), 8, mm.MOE_BF16, max(lengths), p.table.shape[1], 64 ** -0.5
    need = mm.moe_paged_attention_workspace_bytes(c, p.cache.c)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")
    dq = q.cuda()
    other, other_lse = torch.empty_like(dq), torch.empty_like(lse)
    mm.moe_paged_attention(c, p.cache.c, dq, p.table.cuda(), n, other, other_lse, ws, need)
    _check(p, kv, q, other, other_lse)
    assert attn(dq, p.table.cuda(), n, max(lengths), out=dq) is dq and torch.equal(dq, out)


@pytest.mark.parametrize("cache, dim, window", [(BF16, 128, 0), (E4M3, 64, 0), (BF16, 32, 100)])
@pytest.mark.parametrize("sequences, longest", [(70, 300), (130, 64), (130, 500), (130, 65), (290, 130), (33, 700), (520, 130), (290, 40)])
def test_batches_of_many_short_sequences(sequences, longest, cache, dim, window):
    """As many units as run at once and up to several times as many, one a workgroup or shared out, with sequences among them that have nothing."""
    lengths = torch.randint(0, longest + 1, (sequences,), generator=gen(sequences + longest)).tolist()
    lengths[3] = lengths[-1] = 0
    lengths[5] = longest
    _run(lengths, 16, 16, 8, dim, BF16, cache, seed=longest, max_len=longest, window=window)


@pytest.mark.parametrize("sequences, heads, dim, max_len", [(40, 128, 256, 5), (3, 200, 48, 5), (130, 72, 128, 40), (30, 64, 64, 9000)])
def test_wide_rows_without_anything(sequences, heads, dim, max_len):
    """Zeros and NaN in whole rows of many channels, by however many workgroups write them; two sequences have something."""
    lengths = [0] * sequences
    lengths[1], lengths[-1] = 4, max_len
    p = Paged(lengths, 16, 8, dim, BF16, seed=sequences)
    kv = p.fill(1, [0] * sequences)
    given = list(lengths)
    for s in range(2, sequences - 1, 3):
        given[s] = -1 if s % 2 else max_len + 1
    q = torch.randn((sequences, heads, dim), generator=gen(2)).to(BF16)
    out, lse = torch.full((sequences, heads, dim), 7.0, dtype=BF16, device="cuda"), torch.full((sequences, heads), 7.0, device="cuda")
    mm.DecodeAttention(p.cache, heads)(q.cuda(), p.table.cuda(), torch.tensor(given, dtype=torch.int32, device="cuda"), max_len, out=out, lse=lse)
    _check(p, kv, q, out, lse, only=(1, sequences - 1))
    for s, n in enumerate(given):
        if n == 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all(), s
        elif n < 0 or n > max_len:
            assert out[s].isnan().all() and lse[s].isnan().all(), s


@pytest.mark.parametrize("cache", [BF16, E4M3])
def test_offsets_beyond_32_bits(cache):
    """Pages behind 2^32 elements of the cache."""
    far = (1 << 32) // (4 * 64 * 128) + 5
    _run([100, 700], 64, 8, 4, 128, BF16, cache, seed=1, far=far)


def test_refusals():
    p = Paged([20, 3], 16, 2, 32, BF16, seed=1)
    q, table, n = torch.ones((2, 4, 32), dtype=BF16, device="cuda"), p.table.cuda(), torch.tensor([20, 3], dtype=torch.int32, device="cuda")
    attn = mm.DecodeAttention(p.cache, 4)
    for bad in (lambda: attn(q[:, :2], table, n, 20), lambda: attn(q[..., :16], table, n, 20), lambda: attn(q, table[:1], n, 20), lambda: attn(q, table, n[:1], 20),
                lambda: attn(q, table.long(), n, 20), lambda: attn(q, table, n.long(), 20), lambda: attn(q.cpu(), table, n, 20), lambda: attn(q, table.cpu(), n, 20),
                lambda: attn(q, table, n.cpu(), 20), lambda: attn(q, table, n, -1), lambda: attn(q, table, n, 20, out=q.float()), lambda: attn(q, table, n, 20, out=q[:1]),
                lambda: attn(q, table, n, 20, lse=torch.ones((2, 4))), lambda: attn(q, table, n, 20, lse=torch.ones((2, 4), dtype=BF16, device="cuda")),
                lambda: attn(q[:1].expand(2, 4, 32), table, n, 20), lambda: attn(q, table[:1].expand(2, table.shape[1]), n, 20),
                lambda: mm.DecodeAttention(p.cache, 3), lambda: mm.DecodeAttention(p.cache, 0)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: mm.DecodeAttention(p.cache, 4, scale=math.nan)(q, table, n, 20), lambda: mm.DecodeAttention(p.cache, 4, window=-1)(q, table, n, 20),
                lambda: mm.DecodeAttention(p.cache, 4, softcap=-1.0)(q, table, n, 20), lambda: attn(q, table, n, 2 ** 31 - 5)):
        with pytest.raises(mm.MoeError):
            bad()


# ------------------------------------------------------------------------------------ together, graphs, streams
@pytest.mark.parametrize("cache", [BF16, E4M3, FP32])
def test_generation_step_by_step(cache):
    """Prompts of different lengths in chunks, then tokens one by one: appended, attended, checked against all that was appended so far."""
    dtype = FP32 if cache is FP32 else BF16
    B, heads, kv_heads, dim, page = 4, 8, 2, 64, 16
    prompts, steps = [5, 0, 33, 16], 20
    p = Paged([n + steps for n in prompts], page, kv_heads, dim, cache, seed=1)
    rot = mm.Rotary.scaled(dim, layout="interleaved")
    attn = mm.DecodeAttention(p.cache, heads)
    table, g = p.table.cuda(), gen(2)
    have = [0] * B

    def new(n, h):
        return torch.randn((n, h, dim), generator=g).to(dtype).cuda()

    def rows(s, n):
        page_, off = p.slots(s, torch.arange(n))
        page_, off = page_.cuda(), off.cuda()
        pick = lambda t, sc: (t.view(torch.uint8)[page_, :, off].view(E4M3).float().double() * sc[page_, :, off].double()[..., None] if cache is E4M3  # noqa: E731
                              else t[page_, :, off].double()).cpu()
        return pick(p.k, p.k_scale), pick(p.v, p.v_scale)
    seq = torch.tensor([s for s, n in enumerate(prompts) for _ in range(n)], dtype=torch.int32, device="cuda")
    pos = torch.tensor([i for n in prompts for i in range(n)], dtype=torch.int32, device="cuda")
    p.cache.append(new(len(pos), kv_heads), new(len(pos), kv_heads), pos, table, seq=seq, rotary=rot)
    have = list(prompts)
    for _ in range(steps):
        at = torch.tensor(have, dtype=torch.int32, device="cuda")
        q = p.cache.append(new(B, kv_heads), new(B, kv_heads), at, table, rotary=rot, q=new(B, heads))
        have = [n + 1 for n in have]
        out = attn(q, table, at + 1, max(have))
        _check(p, [rows(s, n) for s, n in enumerate(have)], q.cpu(), out, lengths=have)


def test_a_captured_step_replayed_with_other_lengths_pages_and_tokens():
    """One graph of append and attention; every replay against the eager calls on the state it ran on, with eager work between them."""
    lengths = [700, 30, 2500]
    p = Paged([n + 8 for n in lengths], 16, 2, 64, BF16, seed=1)
    p.fill(2)
    rot, attn, eager = mm.Rotary.scaled(64), mm.DecodeAttention(p.cache, 8), mm.DecodeAttention(p.cache, 8)
    most = 3000
    k, v, q = (torch.zeros((3, h, 64), dtype=BF16, device="cuda") for h in (2, 2, 8))
    table, pos, n = p.table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda") + 1
    q_out, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((3, 8), device="cuda")

    def step(a):
        p.cache.append(k, v, pos, table, rotary=rot, q=q, q_out=q_out)
        a(q_out, table, n, most, out=out, lse=lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(attn)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(attn)
    for i in range(5):
        for t, h in ((k, 2), (v, 2), (q, 8)):
            t.copy_(torch.randn((3, h, 64), generator=gen(10 * i + h)).to(BF16))
        if i == 2:                                           # a sequence ends, another one begins in its slot
            pos[1], n[1] = 0, 1
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), q_out.clone()
        attn(q_out, table[:, :300 // 16 * 16], n.clamp(max=300), 300)          # the graph's object in an eager call, another shape
        big = mm.DecodeAttention(p.cache, 8)(q_out.repeat(40, 1, 1), table.repeat(40, 1), n.repeat(40), most)
        attn(q_out.repeat(40, 1, 1), table.repeat(40, 1), n.repeat(40), most)  # its workspace grows
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1]) and torch.equal(q_out, got[2])
        assert torch.isfinite(big).all()
        pos += 1
        n += 1


def test_two_graphs_with_objects_of_their_own_side_by_side():
    lengths = [6000, 100]
    p = Paged(lengths, 16, 2, 128, BF16, seed=1)
    kv = p.fill(2)
    table, n = p.table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    made = []
    for i in range(2):
        q = torch.randn((2, 4, 128), generator=gen(i)).to(BF16)
        attn, dq = mm.DecodeAttention(p.cache, 4), q.cuda()
        out = attn(dq, table, n, 6000).clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            attn(dq, table, n, 6000, out=out)
        made.append((q, dq, attn, out, graph, torch.cuda.Stream()))
    for _ in range(4):
        for m in made:
            m[3].fill_(0)
        torch.cuda.synchronize()
        for m in made:
            with torch.cuda.stream(m[5]):
                m[4].replay()
        torch.cuda.synchronize()
        for m in made:
            _check(p, kv, m[0], m[3])


def test_memory_given_back_while_another_stream_uses_it():
    """Rotation, cache and workspace dropped right after calls that still wait on their stream: tensors made meanwhile keep what is in them, and results
    are right."""
    side = torch.cuda.Stream()
    want = None
    for _ in range(3):
        p = Paged([4000], 16, 2, 64, BF16, seed=1)
        p.fill(2)
        rot, attn = mm.Rotary.scaled(64), mm.DecodeAttention(p.cache, 4)
        k, v, q = (torch.ones((1, h, 64), dtype=BF16, device="cuda") for h in (2, 2, 4))
        table, pos, n = p.table.cuda(), torch.tensor([3999], dtype=torch.int32, device="cuda"), torch.tensor([4000], dtype=torch.int32, device="cuda")
        q_out, out = torch.empty_like(q), torch.empty_like(q)
        attn(q, table, n, 4000, out=out)                     # the workspace belongs to this stream
        sizes = [t.untyped_storage().nbytes() for t in (p.k, p.v, rot.freq, attn.ws)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        p.cache.append(k, v, pos, table, rotary=rot, q=q, q_out=q_out, stream=side)
        attn(q_out, table, n, 4000, out=out, stream=side)
        del p, rot, attn
        made = [torch.full((b,), 55, dtype=torch.uint8, device="cuda") for b in sizes for _ in range(3)]
        torch.cuda.synchronize()
        assert all((t == 55).all() for t in made)
        want = out.clone() if want is None else want
        assert torch.equal(out, want)
