"""Rows without anything to norm: with eps 0 too, a row of zeros stays one, and a token
without routes leaves its residual."""
import pytest
import torch

import block_ref as B
from paper_2609_33385_amd import oled

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTHS = [8, 128, 512, 520, 2048, 4096, 8192, 16384]     # every form


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_in_zero_rows(H, dtype):
    g = torch.Generator().manual_seed(H)
    T, zero = 7, [0, 3, 6]
    x = torch.randn((T, H), generator=g).to(TYPES[dtype])
    x[zero] = 0
    x[3] = -0.0
    w = (1 + 0.1 * torch.randn(H, generator=g)).cuda()

    def call(rows):
        t = rows.shape[0]
        n = torch.full((t, H), 9.0, dtype=TYPES[dtype], device="cuda")
        q = torch.full((t, H), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.full((t, -(-H // 128)), 9.0, device="cuda")
        assert oled.oled_norm_in(rows.cuda(), dtype, H, t, H, w, 0.0, n, q, s) == oled.OLED_OK
        torch.cuda.synchronize()
        return n.cpu(), q.cpu(), s.cpu()
    n, q, s = call(x)
    assert (n[zero] == 0).all() and (q[zero] & 0x7F == 0).all()
    least = torch.tensor(2.0 ** -100) / 448
    assert (s[zero] == least).all()
    keep = [t for t in range(T) if t not in zero]
    for a, b in zip((n, q, s), call(x[keep].contiguous())):      # the others: what they are alone
        assert torch.equal(a[keep].float(), b.float()) and torch.isfinite(b.float()).all()
    v = x[keep].double()
    v = v / v.pow(2).mean(1, keepdim=True).sqrt() * w.cpu().double()
    half = {"f32": B.U, "bf16": 2.0 ** -8}[dtype] * (1 + 2.0 ** -7)
    # the mean square is within (H + 4) U, its root within half that, then three products
    assert torch.all((n[keep].double() - v).abs() <= (half + ((H + 4) / 2 + 8) * B.U) * v.abs())


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("f_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_norm_out_nothing_to_norm(H, k, f_dtype, y_dtype):
    g = torch.Generator().manual_seed(H + k)
    T, zero = 6, [1, 5]
    f = torch.randn((T * max(k, 1), H), generator=g).to(TYPES[f_dtype])
    x = torch.randn((T, H), generator=g).to(TYPES[y_dtype])
    w, gate = (torch.randn((2, H), generator=g) + 2).cuda()
    weights = inv = None
    if k:
        weights = torch.rand((T, k), generator=g).cuda()
        inv = torch.randperm(T * k, generator=g).int().view(T, k)
        f[inv[1].long()] = float("nan")      # read by no route
        inv[1] = -1
        f[inv[5].long()] = 0                 # routes whose rows are zeros
        inv = inv.cuda()
    else:
        f[zero] = 0
    y = torch.full((T, H), 9.0, dtype=TYPES[y_dtype], device="cuda")
    assert oled.oled_norm_out(f.cuda(), f_dtype, weights, inv, k, T, H, w, 0.0, gate, 0, x.cuda(), 0.5, y,
                              y_dtype) == oled.OLED_OK
    torch.cuda.synchronize()
    assert torch.equal(y[zero].cpu(), (0.5 * x[zero].float()).to(TYPES[y_dtype]))
    assert torch.isfinite(y).all()
    # without a residual: zeros
    assert oled.oled_norm_out(f.cuda(), f_dtype, weights, inv, k, T, H, w, 0.0, None, 0, None, 1.0, y,
                              y_dtype) == oled.OLED_OK
    assert (y[zero] == 0).all() and torch.isfinite(y).all()


def test_norm_in_nan_is_not_a_zero_row():
    """A NaN in a row reaches all of the row, with eps 0 as with any."""
    x = torch.zeros((3, 256))
    x[1, 9] = float("nan")
    n = torch.zeros((3, 256), device="cuda")
    w = torch.ones(256, device="cuda")
    assert oled.oled_norm_in(x.cuda(), "f32", 256, 3, 256, w, 0.0, n, None, None) == oled.OLED_OK
    assert torch.isnan(n[1]).all() and (n[0] == 0).all() and (n[2] == 0).all()
