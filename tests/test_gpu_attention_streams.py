"""The attention step's Python calls on a stream given as torch's object or as its handle, with results that they take themselves."""
import threading

import pytest
import torch

from paper_2510_12357_amd import binding as mm
from attention_util import BF16, Paged, gen

pytestmark = pytest.mark.gpu


def _made():
    lengths = [700, 30, 2500]
    p = Paged([n + 1 for n in lengths], 16, 2, 64, BF16, seed=1)
    p.fill(2)
    k, v, q = (torch.randn((3, h, 64), generator=gen(h)).to(BF16).cuda() for h in (2, 2, 8))
    return p, mm.Rotary.scaled(64), mm.DecodeAttention(p.cache, 8), (k, v, q), p.table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("as_handle", [False, True])
def test_a_step_on_a_stream_of_its_own(as_handle):
    p, rot, attn, (k, v, q), table, pos = _made()
    n = pos + 1
    q_want = p.cache.append(k, v, pos, table, rotary=rot, q=q)
    want, turned = attn(q_want, table, n, 2501).clone(), rot(q, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if as_handle else side
    q_out = p.cache.append(k, v, pos, table, rotary=rot, q=q, stream=stream)
    out, again = attn(q_out, table, n, 2501, stream=stream), rot(q, pos, stream=stream)
    side.synchronize()
    assert torch.equal(q_out, q_want) and torch.equal(out, want) and torch.equal(again, turned)


def test_two_threads_with_one_object_of_each():
    """Rotations both ways and attention with two bounds, of one shape each, from two threads on one stream."""
    p, rot, attn, (k, v, q), table, pos = _made()
    n = pos.clone()
    forth, back = rot(q, pos), rot(q, pos, inverse=True)
    short = n.clamp(max=600)
    long_want, short_want = attn(q, table, n, 2501), attn(q, table, short, 600)
    torch.cuda.synchronize()
    wrong = []

    def work(first):
        for _ in range(200):
            turned = rot(q, pos, inverse=not first)
            seen = attn(q, table, n if first else short, 2501 if first else 600)
            if not torch.equal(turned, forth if first else back) or not torch.equal(seen, long_want if first else short_want):
                wrong.append(first)
    threads = [threading.Thread(target=work, args=(f,)) for f in (True, False)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
