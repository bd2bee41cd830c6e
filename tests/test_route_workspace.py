"""The routing workspace of more tokens serves fewer (no GPU)."""
import pytest

from paper_2609_33385_amd import oled

P = 1 << 20     # a pointer that is never read


@pytest.mark.parametrize("E", [1, 64, 256])
def test_workspace_grows_with_tokens(E):
    sizes = [oled.oled_route_scored_workspace(T, E) for T in range(1, 65536)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[0] >= 8 * E and sizes[-1] <= 4 * E * 1100


@pytest.mark.parametrize("T", [8193, 65535])
def test_a_byte_short_is_refused(T):
    r = oled.Router(n_experts=64, top_k=8, n_groups=1, top_groups=1, group_best=1, score=1, renorm=1, dtype=0, scale=1.0)
    short = oled.oled_route_scored_workspace(T, 64) - 1
    got = oled.load().oled_route_scored(r, P, None, None, T, P, P, P, P, P, P, None, P, short, None)
    assert got == oled.OLED_ERR_INVALID_ARG and "workspace" in oled.last_error(None)
