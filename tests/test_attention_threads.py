"""The attention step's Python objects when two threads share one: the interpreter's lock is given up inside of a C call, so that another call of the same shapes can run
while it reads its description.  A stand-in for the library lets that happen every time, without a GPU."""
import contextlib
import os
import threading

import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.skipif(not os.path.exists(mm.LIB_PATH), reason="libmobile_moe.so not built")


class _Library:
    """Whatever a call finds in its description once `meanwhile` has run in another thread."""

    def __init__(self, found):
        self.meanwhile, self.found, self.got = None, found, []

    def call(self, *args):
        other, self.meanwhile = self.meanwhile, None
        if other is not None:
            t = threading.Thread(target=other)
            t.start()
            t.join()
        self.got.append(self.found(*args))
        return 0


@pytest.fixture
def no_gpu(monkeypatch):
    """Host tensors pass for a device's."""
    mm.load_library()
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(mm, "_on_one_gpu", lambda *t: None)
    monkeypatch.setattr(mm, "_raw_stream", lambda stream, device: 0)
    monkeypatch.setattr(mm, "_call_on", lambda device, function, *args: function(*args))
    monkeypatch.setattr(mm._Owner, "_used_on", lambda self, stream, handle: None)

    def library(found, name):
        lib = _Library(found)
        setattr(lib, name, lib.call)
        monkeypatch.setattr(mm, "_lib", lib)
        return lib
    return library


@pytest.mark.parametrize("first", [False, True])
def test_one_rotary_both_ways(no_gpu, first):
    """A forward pass in one thread, the backward pass of another one's in a second."""
    rot = mm.Rotary(torch.ones(4, dtype=torch.float64))
    lib = no_gpu(lambda ref, *args: ref._obj.inverse, "moe_rope")
    x, pos = torch.zeros((3, 2, 8)), torch.zeros(3, dtype=torch.int32)
    for warm in (False, True):                               # also where both directions have been called before
        lib.meanwhile = lambda: rot(x, pos, out=torch.zeros_like(x), inverse=not first)
        rot(x, pos, out=torch.zeros_like(x), inverse=first)
        assert lib.got == [int(not first), int(first)], warm
        lib.got = []


def _attention(monkeypatch, n_heads=2):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _NoStream())
    return mm.DecodeAttention(mm.KvCache.empty(4, 16, 1, 16, device="cpu"), n_heads)


class _NoStream:
    def synchronize(self):
        pass


def test_one_attention_with_two_bounds(no_gpu, monkeypatch):
    """The bound of one thread's lengths does not become the other one's, whose longer sequences would be NaN."""
    attn = _attention(monkeypatch)
    q, table, n = torch.zeros((3, 2, 16)), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    lib = no_gpu(lambda ref, *args: ref._obj.max_len, "moe_paged_attention")
    lib.moe_paged_attention_workspace_bytes = lambda c, cache: 0
    for warm in (False, True):
        lib.meanwhile = lambda: attn(q, table, n, 5, out=torch.zeros_like(q))
        attn(q, table, n, 60, out=torch.zeros_like(q))
        assert lib.got == [5, 60], warm
        lib.got = []
    for bound in (60, 60, 5, 7, 60):                         # each call its own one
        attn(q, table, n, bound, out=torch.zeros_like(q))
    assert lib.got == [60, 60, 5, 7, 60]
    for bound in (-1, 2 ** 31):
        with pytest.raises(ValueError):
            attn(q, table, n, bound, out=torch.zeros_like(q))
    attn(q, table, n, 60, out=torch.zeros_like(q))
    assert lib.got[-1] == 60


def test_one_attention_whose_workspace_grows_in_two_threads(no_gpu, monkeypatch):
    """Each call gets a workspace of its size, whichever of two that grow it at once comes last; none that a call was given is let go."""
    attn = _attention(monkeypatch)
    q, table, n = torch.zeros((3, 2, 16)), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    lib = no_gpu(lambda ref, cache, q, t, n, out, lse, ws, ws_bytes, *args: (ref._obj.max_len, ws, ws_bytes), "moe_paged_attention")
    lib.moe_paged_attention_workspace_bytes = lambda c, cache: 1000 * c._obj.max_len
    empty, other = torch.empty, []

    def slow_empty(*args, **kw):
        """Between a thread's decision for a size and its workspace another one gets its own."""
        if kw.get("dtype") is torch.uint8 and not other:
            other.append(threading.Thread(target=lambda: attn(q, table, n, 60, out=torch.zeros_like(q))))
            other[0].start()
            other[0].join(0.5)                               # or waits for this one
        return empty(*args, **kw)
    monkeypatch.setattr(mm, "_torch_stream", lambda stream, device=None: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch, "empty", slow_empty)
    attn(q, table, n, 5, out=torch.zeros_like(q))
    other[0].join()
    attn(q, table, n, 60, out=torch.zeros_like(q))
    kept = {t.data_ptr(): t.numel() for t in [attn.ws] + attn._outgrown}
    assert len(lib.got) == 3
    for max_len, ws, ws_bytes in lib.got:
        assert ws in kept and ws_bytes >= 1000 * max_len and kept[ws] == ws_bytes, (max_len, ws_bytes, kept)


def test_what_an_object_was_made_with_stays(no_gpu, monkeypatch):
    """Calls keep their descriptions, so that another window or scale would count for some shapes and not for others: it is an object of its own."""
    attn, rot = _attention(monkeypatch), mm.Rotary(torch.ones(4, dtype=torch.float64), mscale=2.0)
    assert (attn.scale, attn.window, attn.softcap, attn.n_heads) == (0.25, 0, 0.0, 2) and (rot.layout, rot.mscale, rot.rotary_dim) == ("half", 2.0, 8)
    for thing, names in ((attn, ("scale", "window", "softcap", "n_heads", "cache")), (rot, ("layout", "mscale", "rotary_dim", "freq"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(thing, name, getattr(thing, name))
