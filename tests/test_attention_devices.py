"""Streams of the attention step's Python objects whose tensors are on another device than the current one.  Stand-ins, without a GPU."""
import os
import threading

import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.skipif(not os.path.exists(mm.LIB_PATH), reason="libmobile_moe.so not built")
ONE, TWO = torch.device("cuda", 0), torch.device("cuda", 1)


class _Stream:
    def __init__(self, device, handle):
        self.device, self.cuda_stream = device, handle


@pytest.fixture
def two_devices(monkeypatch):
    """Device 0 is the current one; each has its own current stream."""
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream(ONE if device is None else torch.device(device), 0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: _Stream(ONE if device is None else torch.device(device), handle))
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)


class _Tensor:
    shape, dtype = torch.Size((2, 1, 16)), torch.float32

    def __init__(self, device):
        self.device, self.recorded = device, []

    def record_stream(self, stream):
        self.recorded.append((stream.device, stream.cuda_stream))


@pytest.mark.parametrize("given, handle", [(None, 0), (77, 77), (_Stream(TWO, 55), 55)])
def test_memory_is_recorded_on_its_own_device(two_devices, given, handle):
    class Owner(mm._Owner):
        memory = (_Tensor(TWO), None, _Tensor(TWO))

        def _memory(self):
            return self.memory
    owner = Owner()
    for _ in range(2):
        owner._used_on(given, handle)
    assert [t.recorded for t in owner.memory if t is not None] == [[(TWO, handle)]] * 2


@pytest.mark.parametrize("call", ["rotary", "append", "attention", "workspace"])
@pytest.mark.parametrize("given", [None, 77])
def test_results_are_taken_on_their_own_device(two_devices, monkeypatch, call, given):
    """New tensors belong to the stream that writes them, of the device that they are on."""
    entered = []

    class Entered:
        def __init__(self, stream):
            entered.append((stream.device, stream.cuda_stream))

        def __enter__(self):
            pass

        def __exit__(self, *args):
            pass

    class Made(Exception):
        pass

    def empty(*args, device=None, **kw):
        assert torch.device(device) == TWO
        raise Made
    monkeypatch.setattr(torch.cuda, "stream", Entered)
    monkeypatch.setattr(torch, "empty", empty)
    x = _Tensor(TWO)
    with pytest.raises(Made):
        if call == "rotary":
            mm.Rotary.__call__(mm.Rotary.__new__(mm.Rotary), x, None, stream=given)
        elif call == "append":
            mm.KvCache.append(mm.KvCache.__new__(mm.KvCache), x, x, None, None, q=x, stream=given)
        else:
            attn = mm.DecodeAttention.__new__(mm.DecodeAttention)
            attn.ws, attn._growing = None, threading.Lock()
            attn._cache = type("Cache", (), {"k": x})
            if call == "attention":
                attn(x, None, None, 1, stream=given)
            else:
                attn._workspace(1, given)
    assert entered == [(TWO, given or 0)]
