"""The chained block as its callers use it: any number of tokens up to its most, and
refused calls."""
import pytest
import torch

import test_gpu_block8 as T8
from paper_2609_33385_amd import block8, oled

pytestmark = pytest.mark.gpu
H = T8.SMALL.hidden


def inputs(T, seed=0):
    g = torch.Generator().manual_seed(1000 * seed + T)
    return [torch.randn((T, H), generator=g).bfloat16().cuda() for _ in range(2)]


def test_fewer_tokens_than_laid_out():
    """A block for many tokens gives what one laid out for the call's own number gives."""
    block = block8.make_block(T8.SMALL, 5, 9000, 16)
    for T in (8192, 100, 9000, 8193, 1):
        own = block8.make_block(T8.SMALL, 5, T, 16)
        x, attn = inputs(T)
        y = x.clone()
        own.forward(x, attn)
        block.forward(y, attn)
        torch.cuda.synchronize()
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        assert torch.isfinite(x.float()).all()


def test_refused_call_leaves_x():
    block = T8.made()
    router = oled.Router(n_experts=16, top_k=4, n_groups=3, top_groups=1, group_best=1, score=0, renorm=1, scale=1.0)
    other = block8.Block8(router, H, T8.SMALL.inter, 4, block.w_out, block.w_gate, block.experts)
    x, attn = inputs(4)
    y = x.clone()
    with pytest.raises(oled.OledError, match="oled_route_scored"):
        other.forward(y, attn)
    torch.cuda.synchronize()
    assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def busy(stream, products=12):
    """Some ten milliseconds of work on a stream."""
    with torch.cuda.stream(stream):
        a = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
        for _ in range(products):
            a = a @ a
    return a


def test_first_call_follows_the_making():
    """Weights that the making stream is still writing are whole when the first call, on
    another stream, reads them."""
    base = T8.made()
    T = 64
    x, attn = inputs(T, 3)
    want = base.forward(x.clone(), attn)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = [[torch.zeros_like(t) for t in pair] for pair in (base.w_out, base.w_gate)]
    torch.cuda.synchronize()
    keep = busy(torch.cuda.current_stream())
    for pair, whole in zip(late, (base.w_out, base.w_gate)):
        for t, w in zip(pair, whole):
            t.view(torch.uint8).copy_(w.view(torch.uint8))
    block = block8.Block8(base.router, H, T8.SMALL.inter, T, tuple(late[0]), tuple(late[1]), base.experts, None, base.bias,
                          base.norm_in, base.norm_attn, base.norm_out)
    block.forward(x, attn, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(x.view(torch.int16), want.view(torch.int16))
    del keep


def test_calls_on_streams_in_turn():
    """Calls on several streams with nothing waiting between them are as those alone, and
    a block that goes away leaves its memory only after its last call."""
    base = T8.made()
    sets = [inputs(T, 7 + i) for i, T in enumerate((160, 3, 97, 160))]
    want = []
    for x, attn in sets:
        want.append(base.forward(x.clone(), attn))
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for rep in range(4):
        block = block8.make_block(T8.SMALL, 5, 160, 16)
        xs = [x.clone() for x, _ in sets]
        torch.cuda.synchronize()
        keep = busy(streams[rep % 3], 3)
        for i, x in enumerate(xs):
            block.forward(x, sets[i][1], stream=streams[(rep + i) % 3])
        sizes = [t.numel() for t in (block.q, block.x1, block.routed, block.expert_ws)]
        del block
        junk = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
        torch.cuda.synchronize()
        for x, y in zip(xs, want):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        del junk, keep


def test_stream_by_handle_and_graphs_between():
    """A stream given by its handle; a graph of the block recorded on a stream that made no
    call, replayed between calls on another."""
    block = T8.made()
    T = 40
    (x, attn), (x2, attn2) = inputs(T, 1), inputs(T, 2)
    want, want2 = block.forward(x.clone(), attn), block.forward(x2.clone(), attn2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = x.clone()
    torch.cuda.synchronize()
    block.forward(y, attn, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(y.view(torch.int16), want.view(torch.int16))
    graph, z = torch.cuda.CUDAGraph(), x.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        block.forward(z, attn)
    for _ in range(3):
        z.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z.view(torch.int16), want.view(torch.int16))
        y2 = x2.clone()
        torch.cuda.synchronize()
        block.forward(y2, attn2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(y2.view(torch.int16), want2.view(torch.int16))
