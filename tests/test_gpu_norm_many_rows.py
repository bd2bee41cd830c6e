"""Norms of more rows than one launch takes threads for."""
import pytest
import torch

from paper_2609_33385_amd import oled

pytestmark = pytest.mark.gpu


# a wavefront a row (four rows a workgroup) and a workgroup a row
@pytest.mark.parametrize("T,H", [((1 << 25) + 5, 8), ((1 << 26) + 9, 8), ((1 << 23) + 1, 520), ((1 << 24) + 3, 520)])
def test_rows_past_a_launch(T, H):
    """Each row holds its number (modulo 251): all are where they belong."""
    v = (torch.arange(T, device="cuda") % 251 - 125).bfloat16()
    x = v[:, None].expand(T, H).contiguous()
    n = torch.full((T, H), 300.0, dtype=torch.bfloat16, device="cuda")
    assert oled.oled_norm_in(x, "bf16", H, T, H, None, 0.0, n, None, None) == oled.OLED_OK
    assert torch.equal(n, x)
    del n
    # one route a token, of every second row; a gate row for every 2^20 tokens
    k = 1 if H == 8 else 0
    weights = inv = None
    if k:
        weights = torch.full((T,), 2.0, device="cuda")
        inv = torch.where(torch.arange(T, device="cuda") % 2 == 0, torch.arange(T, device="cuda"), -1).int()
    gate = torch.ones((-(-T // (1 << 20)), H), device="cuda")
    gate[-1] = 4
    y = torch.full((T, H), 300.0, dtype=torch.bfloat16, device="cuda")
    assert oled.oled_norm_out(x, "bf16", weights, inv, k, T, H, None, 0.0, gate, 1 << 20, None, 0.0, y,
                              "bf16") == oled.OLED_OK
    want = v.float()
    if k:
        want *= 2
        want[1::2] = 0
    want[(T - 1) // (1 << 20) * (1 << 20):] *= 4
    assert torch.equal(y, want.bfloat16()[:, None].expand(T, H))
