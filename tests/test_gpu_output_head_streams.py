"""The output head's Python objects in graphs and on several streams: memory that a graph or another stream still uses is not given away."""
import pytest
import torch

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


@pytest.mark.parametrize("T, K", [(40, 512), (100, 333)])
def test_a_graph_outlives_larger_calls_of_its_object(T, K):
    """Captured with few tokens, then eager prompts on the same object and tensors that take whatever memory is free: the replays write over
    none of them and are right."""
    N = 700
    weight = torch.randn((N, K), generator=_gen(1)).cuda()
    lin, other = mm.Int8Linear.quantize(weight), mm.Int8Linear.quantize(weight)
    x = torch.zeros((T, K), dtype=BF16, device="cuda")
    out = torch.empty((T, N), dtype=FP32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lin(x, out=out)
    torch.cuda.synchronize()
    size = lin.ws.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lin(x, out=out)
    for i in range(4):
        prompt = torch.randn((T * (i + 2) ** 2, K), generator=_gen(i)).cuda()
        assert torch.equal(lin(prompt), other(prompt))
        assert lin.ws.numel() > size
        with torch.cuda.stream(side):
            there = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(40)]
        here = [torch.full((size,), 9, dtype=torch.uint8, device="cuda") for _ in range(40)]
        torch.cuda.synchronize()
        x.copy_(torch.randn((T, K), generator=_gen(10 + i)).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other(x))
        assert all((t == 7).all() for t in there) and all((t == 9).all() for t in here)


def test_codes_made_on_another_stream_take_no_memory_of_this_one():
    """A tensor that this stream still has to read, given back already: its memory is not what a side stream's codes are written to."""
    rows, K = 64, 1024
    x = torch.randn((rows, K), generator=_gen(0)).cuda()
    want = mm.quantize_rows(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        last = [torch.full((rows * K,), 77, dtype=torch.int8, device="cuda") for _ in range(20)]
        torch.cuda._sleep(20_000_000)
        copies = [t.clone() for t in last]
        del last
        q, s = mm.quantize_rows(x, stream=side)
        lin = mm.Int8Linear.quantize(x, stream=side)
        torch.cuda.synchronize()
        assert all((t == 77).all() for t in copies)
        assert torch.equal(q, want[0]) and torch.equal(s, want[1]) and torch.equal(lin.w, q) and torch.equal(lin.w_scale, s)


@pytest.mark.parametrize("T, V", [(3, 131072), (300, 4000)])
def test_buffers_given_back_while_another_stream_fills_them(T, V):
    """Dropped right after the call, which still waits on its stream: tensors made meanwhile keep what is in them."""
    z = (torch.randn((T, V), generator=_gen(0)) * 3).cuda()
    tokens = torch.zeros((T, 2), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        b = mm.LogprobBuffers(T, 2, 20, V)
        kinds = [(t.numel(), t.dtype) for t in (b.token_logp, b.entropy, b.conf, b.top_idx, b.top_logp, b.ws)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        b.run(z, tokens, stream=side)
        del b
        made = [torch.full((n,), 55, dtype=dtype, device="cuda") for n, dtype in kinds for _ in range(4)]
        torch.cuda.synchronize()
        assert all((t == 55).all() for t in made)


def test_weights_given_back_while_another_stream_reads_them():
    """The same of a projection: its codes, scales, bias and workspace."""
    N, K, T = 4000, 1000, 70
    x = torch.randn((T, K), generator=_gen(1)).cuda()
    weight, bias = torch.randn((N, K), generator=_gen(2)).cuda(), torch.randn((N,), generator=_gen(3)).cuda()
    want = mm.Int8Linear.quantize(weight, bias)(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        lin = mm.Int8Linear.quantize(weight, bias.clone())
        lin(x)                                               # the workspace belongs to this stream
        kinds = [t.untyped_storage().nbytes() for t in (lin.w, lin.w_scale, lin.bias, lin.ws)]
        out = torch.empty((T, N), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        lin(x, out=out, stream=side)
        del lin
        made = [torch.full((n,), 55, dtype=torch.uint8, device="cuda") for n in kinds for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all((t == 55).all() for t in made)
