"""What the header promises of the 8-bit packing (no GPU)."""
import pytest

from paper_2609_33385_amd import oled


@pytest.mark.parametrize("H,I", [(16512, 128), (128, 16512), (32768, 32768), (1 << 30, 128), (0, 128), (128, 0), (192, 128)])
def test_bytes_of_unsupported_shapes(H, I):
    assert oled.oled_fp8_expert_bytes(H, I) == 0


def test_bytes_of_the_largest_shape():
    assert oled.oled_fp8_expert_bytes(16384, 16384) == 3 * 2 ** 28 + 12 * 2 ** 14
