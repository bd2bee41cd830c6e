"""Products of more tiles than a launch takes are refused on the host."""
import pytest

from paper_2609_33385_amd import oled

P = 1 << 20     # a pointer that is never read: the refusal comes before a launch


# one row in tiles of 256 features; far apart rows in tiles of 16 x 16
@pytest.mark.parametrize("M,N,lda,ldb", [(1, (1 << 31) - 1, 16, 16), (1, (1 << 31) - 255, 16, 16),
                                         (257, 1 << 30, 16, 16), (16, 1 << 27, 1 << 23, 16),
                                         (1 << 27, 16, 16, 1 << 23), (1 << 16, 1 << 15, 1 << 23, 16)])
def test_too_many_tiles(M, N, lda, ldb):
    got = oled.load().oled_fp8_matmul(P, P, lda, P, P, ldb, M, N, 16, P, N, None)
    assert got == oled.OLED_ERR_UNSUPPORTED
    assert "more tiles than a launch takes" in oled.last_error(None)
