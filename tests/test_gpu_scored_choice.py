"""oled_route_scored without a bias: with group_best 2 the choice is by the score, also
where all groups compete, so saturated scores tie and the lowest ids win; with
group_best 1 it is by the logit."""
import pytest
import torch

import block_ref as B
import test_gpu_scored as S

pytestmark = pytest.mark.gpu


def saturated(T, E, seed):
    """Rising logits whose fp32 sigmoids are all 1 (even tokens) or all 0 (odd ones)."""
    g = torch.Generator().manual_seed(seed)
    l = torch.sort(20 + 60 * torch.rand((T, E), generator=g), dim=1)[0]
    l[1::2] -= 200
    return l


# one workgroup, chunks of 16 and of 64, lanes that load their own rows
@pytest.mark.parametrize("T", [1, 5, 64, 130, 700, 9000])
@pytest.mark.parametrize("E,k,G", [(64, 8, 1), (256, 8, 8), (128, 16, 4), (60, 4, 4), (200, 6, 2), (256, 8, 32),
                                   (16, 16, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_choice_of_saturated_scores(T, E, k, G, dtype):
    l = saturated(T, E, T + E).to(dtype)
    got = S.call(l, None, None, E, k, G, G, 2, "sigmoid", True, 1.0)
    assert torch.equal(got["idx"], torch.arange(k, dtype=torch.int32).expand(T, k))
    assert torch.allclose(got["weights"][::2], torch.full((1,), 1 / k))
    zeros = S.call(l, torch.zeros(E), None, E, k, G, G, 2, "sigmoid", True, 1.0)
    for name in ("idx", "weights", "counts", "offsets", "perm", "inv"):
        assert torch.equal(got[name], zeros[name])
    by_logit = S.call(l, None, None, E, k, G, G, 1, "sigmoid", True, 1.0)
    want = torch.sort(l.double(), dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(by_logit["idx"], want.int())


@pytest.mark.parametrize("T", [7, 500])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_choice_of_ordinary_scores(T, score):
    """Where scores are distinct and 32 bits tell them apart, both rules choose alike."""
    E, k, G = 128, 8, 4
    g = torch.Generator().manual_seed(T)
    # a ramp in another order for each token: neighbours differ by 1/32 of a logit
    order = torch.rand((T, E), generator=g).argsort(1)
    l = (order.float() - 64) / 32
    idx, w, _, _ = B.route(l, torch.zeros(E), None, E, k, G, G, 2, score == "softmax", True, 1.0)
    for best in (1, 2):
        got = S.call(l, None, None, E, k, G, G, best, score, True, 1.0)
        assert torch.equal(got["idx"], idx.int())
        assert torch.all((got["weights"].double() - w).abs() <= (64 + E + 8) * B.U * w)
