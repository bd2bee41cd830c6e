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
