"""What the output head's Python calls refuse of tensors before anything is enqueued (no GPU needed: each refusal comes before the library)."""
import contextlib
import ctypes
import os
import weakref

import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.skipif(not os.path.exists(mm.LIB_PATH), reason="libmobile_moe.so not built")


def _codes(rows, K=64):
    return torch.ones((rows, K), dtype=torch.int8)


# ------------------------------------------------------------------------------------ rows that lie on each other
@pytest.mark.parametrize("step", [0, 1, 63])
def test_rows_of_one_place_are_not_dense_rows(step):
    """A distance of 0 means "dense" to the C calls, so rows that share memory (expanded tensors) must not reach them."""
    x, w, out = torch.zeros((4, 64)), _codes(8), torch.zeros((4, 8))
    lie = lambda t: t.reshape(-1).as_strided(t.shape, (min(step, t.shape[1] - 1), 1))  # noqa: E731
    assert mm.int8_config(x, w, out).ldx == 64
    for a in ((lie(x), w, out), (x, lie(w), out), (x, w, lie(out))):
        with pytest.raises(ValueError, match="rows"):
            mm.int8_config(*a)
    with pytest.raises(ValueError, match="rows"):
        mm.moe_quantize_rows(lie(x), _codes(4), torch.zeros(4))
    with pytest.raises(ValueError, match="rows"):
        mm.LogprobBuffers(4, 0, 1, 64, device="cpu").run(lie(x))


def test_expanded_rows():
    x, w = torch.zeros((1, 64)).expand(4, 64), _codes(1).expand(8, 64)
    for a in ((x, _codes(8), torch.zeros((4, 8))), (torch.zeros((4, 64)), w, torch.zeros((4, 8))),
              (torch.zeros((4, 64)), _codes(8), torch.zeros((1, 8)).expand(4, 8))):
        with pytest.raises(ValueError, match="rows"):
            mm.int8_config(*a)
    for z in (torch.zeros((1, 5)).expand(3, 5), torch.zeros((1, 1)).expand(3, 1)):
        with pytest.raises(ValueError, match="rows"):
            mm.LogprobBuffers(3, 0, 1, z.shape[1], device="cpu").run(z)


def test_a_single_row_may_have_any_stride():
    """A dimension of one row has no distance to a next one."""
    for step in (0, 1, 64, 80):
        c = mm.int8_config(torch.zeros(80).as_strided((1, 64), (step, 1)), _codes(8), torch.zeros((1, 8)).as_strided((1, 8), (step, 1)))
        assert c.ldx >= 64 and c.ldo >= 8
    c = mm.int8_config(torch.zeros((0, 64)), _codes(8), torch.zeros((0, 8)))
    assert (c.T, c.ldx, c.ldo) == (0, 64, 8)


# ------------------------------------------------------------------------------------ workspaces
def test_a_workspace_lives_as_long_as_its_object(monkeypatch):
    """A captured graph holds the address of the workspace that its call had, so a larger call must not give that memory back; and what is
    kept stays below what the largest call took."""
    monkeypatch.setattr(mm, "_torch_stream", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    lin = mm.Int8Linear(_codes(8), torch.ones(8))
    held, largest = [], 0
    for need in list(range(256, 40000, 256)) + [100, 5000, 10 ** 6, 512]:
        address = lin._workspace(need, None)
        largest = max(largest, need)
        assert lin.ws.data_ptr() == address and lin.ws.numel() >= need
        if not any(h() is lin.ws for h in held):
            held.append(weakref.ref(lin.ws))
    assert len(held) > 2 and all(h() is not None for h in held)
    assert sum(h().numel() for h in held) <= 4 * largest


# ------------------------------------------------------------------------------------ devices
def test_host_tensors_are_refused():
    """A kernel would take a host address as it is."""
    lin = mm.Int8Linear(_codes(8), torch.ones(8))
    for x, scale in ((torch.zeros((2, 64)), None), (_codes(2), torch.ones(2)), (_codes(2), torch.ones(2, device="meta"))):
        with pytest.raises(ValueError, match="device"):
            lin(x, x_scale=scale, out=torch.zeros((2, 8)))
    for n, tokens in ((0, None), (1, torch.zeros((2, 1), dtype=torch.int32)), (1, torch.zeros((2, 1), dtype=torch.int32, device="meta"))):
        with pytest.raises(ValueError, match="device"):
            mm.LogprobBuffers(2, n, 1, 64, device="cpu").run(torch.zeros((2, 64)), tokens)


def test_host_tensors_are_refused_by_every_call():
    x, w, out, f = torch.zeros((2, 64)), _codes(8), torch.zeros((2, 8)), torch.zeros(8)
    b = mm.LogprobBuffers(2, 0, 1, 64, device="cpu")
    for call in (lambda: mm.moe_quantize_rows(x, _codes(2), f[:2]), lambda: mm.quantize_rows(x),
                 lambda: mm.moe_matmul_int8(mm.int8_config(_codes(2), w, out), _codes(2), f[:2], w, f, None, out),
                 lambda: mm.moe_linear_int8(mm.int8_config(x, w, out), x, w, f, f, out, torch.zeros(512, dtype=torch.uint8), 512),
                 lambda: mm.moe_token_logprobs(b.c[mm.MOE_FP32], x, None, None, b.entropy, b.conf, b.top_idx, b.top_logp, b.ws, 0)):
        with pytest.raises(ValueError, match="device"):
            call()


# ------------------------------------------------------------------------------------ streams
def test_codes_are_allocated_on_the_stream_that_writes_them(monkeypatch):
    """Memory of another stream may still be read there by earlier work."""
    stack, places, empty = ["current"], [], torch.empty

    @contextlib.contextmanager
    def on(stream):
        stack.append(stream)
        yield
        stack.pop()
    monkeypatch.setattr(mm, "_on_one_gpu", lambda *tensors: None)
    monkeypatch.setattr(mm, "_torch_stream", lambda stream: stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(mm, "moe_quantize_rows", lambda x, q, scale, stream: places.append(stream))
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (places.append(stack[-1]), empty(*a, **k))[1])
    for make in (lambda s: mm.quantize_rows(torch.zeros((3, 20)), s), lambda s: mm.Int8Linear.quantize(torch.zeros((3, 20)), stream=s)):
        places.clear()
        make("side")
        assert places == ["side"] * 3


def test_logprob_buffers_are_known_to_every_stream_that_uses_them(monkeypatch):
    """Once per stream: their memory must not be given away while that stream still works on it."""
    b = mm.LogprobBuffers(3, 2, 4, 131072, device="cpu")
    seen = []
    monkeypatch.setattr(mm, "_torch_stream", lambda stream: stream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: seen.append((t.data_ptr(), stream)))
    for handle, stream in ((5, "a"), (5, "a"), (6, "b"), (5, "a")):
        b._used_on(stream, handle)
    tensors = {t.data_ptr() for t in (b.token_logp, b.entropy, b.conf, b.top_idx, b.top_logp, b.ws)}
    assert len(tensors) == 6 and sorted(seen) == sorted((t, s) for t in tensors for s in ("a", "b"))


def test_weights_and_workspace_are_known_to_every_stream_that_uses_them(monkeypatch):
    lin, seen = mm.Int8Linear(_codes(8), torch.ones(8), torch.ones(8)), []
    monkeypatch.setattr(mm, "_torch_stream", lambda stream: stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: seen.append((t.data_ptr(), stream)))
    for need in (512, 4096):                                 # a larger workspace is another tensor
        seen.clear()
        tensors = {t.data_ptr() for t in (lin.w, lin.w_scale, lin.bias)} | {lin._workspace(need, "a")}
        for handle, stream in ((5, "a"), (5, "a"), (6, "b"), (5, "a")):
            lin._used_on(stream, handle)
        assert sorted(seen) == sorted((t, s) for t in tensors for s in ("a", "b"))


# ------------------------------------------------------------------------------------ rows far apart
def _far(rows, n, step, dtype=torch.float32):
    """Shape and strides of such rows, without their memory."""
    return torch.empty_strided((rows, n), (step, 1), dtype=dtype, device="meta")


@pytest.mark.parametrize("step", [1 << 22, 1024 * 4096 + 3, 1 << 33])
def test_float_tokens_lie_as_far_apart_as_they_like(step):
    """hidden[:, -1] of a batch of prompts: only rows of codes, weights and outputs have to be near each other."""
    c = mm.int8_config(_far(4, 64, step), _codes(8), torch.zeros((4, 8)))
    assert c.ldx == step and mm.moe_linear_int8_workspace_bytes(c) > 0
    P = 1 << 20                                               # an address that passes the alignment checks and is never read
    lib = mm.load_library()
    assert lib.moe_linear_int8(ctypes.byref(c), P, P, P, None, P, None, 0, None) == -6      # MOE_E_WORKSPACE: all else is as it should be
    assert lib.moe_matmul_int8(ctypes.byref(c), P, P, P, P, None, P, None) == -3            # MOE_E_UNSUPPORTED as codes


@pytest.mark.parametrize("step", [1 << 22, 1 << 33])
def test_one_row_has_no_next_one(step):
    """The only row of a tensor whose strides are those of a larger one."""
    c = mm.int8_config(_far(1, 60, step, torch.int8), _far(1, 60, step, torch.int8), _far(1, 1, step))
    assert mm.load_library().moe_matmul_int8(ctypes.byref(c), None, None, None, None, None, None, None) == -1   # past the checks of distances
    assert "x is NULL" in mm.moe_last_error()


def test_rows_far_apart_are_made_dense_for_the_calls_that_need_it():
    near = _far(4, 64, 4096)
    assert mm._near_rows(near, None) is near and mm._near_rows(_far(1, 64, 1 << 30), None).shape == (1, 64)


def test_dense_copies_of_rows_far_apart(monkeypatch):
    streams = []
    monkeypatch.setattr(mm, "_torch_stream", lambda stream: stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: (streams.append(stream), contextlib.nullcontext())[1])
    mem = torch.zeros((1 << 22) + 10)
    mem[0], mem[1 << 22] = 1.0, 2.0
    z = mem.as_strided((2, 10), (1 << 22, 1))
    dense = mm._near_rows(z, "side")
    assert torch.equal(dense, z) and dense.is_contiguous() and streams == ["side"]


# ------------------------------------------------------------------------------------ codes and scales of other forms
@pytest.mark.parametrize("q, scale", [(torch.zeros((4, 64)), torch.zeros(4)), (torch.zeros((4, 64), dtype=torch.int8), torch.zeros(3)),
                                      (torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4, dtype=torch.bfloat16)),
                                      (torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4, dtype=torch.float64)),
                                      (torch.zeros(4 * 64, dtype=torch.int8).reshape(4, 8, 8), torch.zeros(4)),
                                      (torch.zeros((3, 64), dtype=torch.int8), torch.zeros(4))])
def test_codes_and_scales_have_a_place_each(q, scale):
    """The kernel writes a scale of fp32 per row and rows of q.shape[1] codes, whatever stands there."""
    with pytest.raises(ValueError, match="codes|scales"):
        mm.moe_quantize_rows(torch.zeros((4, 60)), q, scale)
