"""Scales of the 8-bit products over all counts of 128s of K: whole and short chunks of
8 in every form. What lies around a caller's scales is NaN and must not matter."""
import pytest
import torch

import test_gpu_fp8 as F
from paper_2609_33385_amd import oled

pytestmark = pytest.mark.gpu


def amid_nan(t):
    """The values of t on the device, in a row with NaN on either side."""
    room = torch.full((t.numel() + 64,), float("nan"), device="cuda")
    room[32: 32 + t.numel()] = t.reshape(-1)
    return room[32: 32 + t.numel()]


# one group of 16 x 16 tiles, 64 x 64 with three and with two ring slots, tiles of 128 and of 256 rows
@pytest.mark.parametrize("M,N", [(33, 192), (300, 640), (1030, 2050), (1030, 4096), (2177, 4100)])
@pytest.mark.parametrize("blocks", [1, 2, 7, 8, 9, 12, 15, 16, 17, 33])
@pytest.mark.parametrize("tail", [128, 48])
def test_matmul_scale_chunks(M, N, blocks, tail):
    """Small integers times powers of two: every product, sum and scale is exact, so the
    result is the rounding of the true one, and one wrong scale shows."""
    K, kb = 128 * (blocks - 1) + tail, blocks
    g = torch.Generator(device="cuda").manual_seed(M + 64 * blocks + tail)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda").float()
    a, b = ints(-2, 3, M, K), ints(-2, 3, N, K)
    a_s, b_s = 2 ** ints(0, 4, M, kb), 2 ** ints(-3, 1, -(-N // 128), kb)
    c = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    aq, bq = (t.to(torch.float8_e4m3fn) for t in (a, b))
    st = oled.oled_fp8_matmul(aq, amid_nan(a_s), K, bq, amid_nan(b_s), K, M, N, K, c, N,
                              torch.cuda.current_stream())
    assert st == oled.OLED_OK, oled.last_error(None)
    va = a.double() * a_s.double().repeat_interleave(128, 1)[:, :K]
    vb = b.double() * b_s.double().repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N]
    assert torch.equal(c, (va @ vb.t().contiguous()).float().bfloat16())


@pytest.mark.parametrize("T,k,E", [(3, 2, 4), (60, 4, 8), (300, 2, 6), (700, 2, 2)])
@pytest.mark.parametrize("H,I", [(128, 1152), (1152, 128), (1024, 1408), (1536, 1024)])
def test_experts_scale_chunks(T, k, E, H, I):
    F.check_experts(T, k, E, H, I)
