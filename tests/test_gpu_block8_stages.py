"""The chained block stage by stage: each buffer that a call leaves against the 64-bit
reference of what the buffers before it hold, within the bounds of the call's own
tests. So a wrong operand, stride, bias, weight or order between two calls shows."""
import pytest
import torch

import block_ref as B
import test_gpu_block8 as T8
import test_gpu_fp8 as F
from paper_2609_33385_amd import block8, oled
from paper_2609_33385_amd import workload as W

pytestmark = pytest.mark.gpu
HALF = F.HALF       # rounding to bf16
EPS = 1e-6
_made = {}


def made(w, slots):
    """A block with a bias that moves choices and norm weights that are not 1; with slots,
    experts share blocks through the slot table."""
    key = (w.n_experts, slots)
    if key not in _made:
        g = torch.Generator().manual_seed(21)
        E, H = w.n_experts, w.hidden
        bias = 0.01 * torch.randint(-12, 13, (E,), generator=g).float()
        router = oled.Router(n_experts=E, top_k=w.top_k, n_groups=4, top_groups=2, group_best=2,
                             score=oled.SCORES["sigmoid"], renorm=1, scale=2.5)
        block = block8.make_block(w, 5, 160, slots, router, bias.cuda())
        block.norm_in.mul_(1 + 0.2 * torch.rand(H, generator=g).cuda())
        block.norm_attn.copy_(1 + 0.2 * torch.randn(H, generator=g).cuda())
        block.norm_out.copy_(1 + 0.2 * torch.randn(H, generator=g).cuda())
        torch.cuda.synchronize()
        _made[key] = block
    return _made[key]


def product(q, s, w):
    """(q o s) W^T in 64 bits, and the bound of oled_fp8_matmul's own test."""
    a, b = B.values(q, s), B.values(*(t.cpu() for t in w), 128)
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    return ref, (a.shape[1] + 16) * B.U * mag + B.cuts(a, b) + HALF * ref.abs() + 1e-37


def normed(f, mag, k, w):
    """f rsqrt(mean f^2 + eps) w and its bound but for the last rounding, as in the test of oled_norm_out."""
    H = f.shape[1]
    gain = w.double().cpu() / torch.sqrt(f.pow(2).mean(1, keepdim=True) + EPS)
    row = mag.pow(2).mean(1, keepdim=True).sqrt() / (f.pow(2).mean(1, keepdim=True) + EPS).sqrt()
    rel = (k + 2) * B.U * mag + (((H + 4) / 2 + 8) * B.U + (k + 2) * B.U * row) * f.abs()
    return f * gain, rel * gain.abs()


def inside(got, ref, bound, what):
    err = (got.double() - ref).abs()
    assert torch.all(err <= bound), (what, float((err / bound).max()))


WIDE = W.Workload(8, "wide-bf16", "bf16", 1, 32, 32, 6, 384, 256, 1, 1, 16)


@pytest.mark.parametrize("w,slots", [(T8.SMALL, 16), (T8.SMALL, 5), (WIDE, 32)])
@pytest.mark.parametrize("T", [1, 2, 33, 160])
def test_stages(w, slots, T):
    E, H, k = w.n_experts, w.hidden, w.top_k
    block = made(w, slots)
    g = torch.Generator().manual_seed(100 + T)
    x = torch.randn((T, H), generator=g).bfloat16()
    attn = torch.randn((T, H), generator=g).bfloat16()
    mask = torch.rand(T, generator=g) < 0.8
    mask[0] = True
    gate = torch.rand((-(-T // 32), H), generator=g)
    y, at = x.clone().cuda(), attn.cuda()
    block.forward(y, at, mask.cuda(), gate.cuda(), 32, 0.75)
    torch.cuda.synchronize()
    got = {n: getattr(block, n)[:T].cpu() for n in ("q", "q_scale", "f", "x1", "logits", "topk_idx", "weights")}
    q1, s1 = torch.zeros((T, H), dtype=torch.uint8, device="cuda"), torch.zeros((T, H // 128), device="cuda")
    assert oled.oled_norm_in(at, "bf16", H, T, H, None, EPS, None, q1, s1) == oled.OLED_OK
    torch.cuda.synchronize()

    # the attention's projection, and its norm onto the residual
    ref, bound = product(q1.cpu().view(B.F8), s1.cpu(), block.w_out)
    inside(got["f"], ref, bound, "f")
    f = got["f"].double()
    n, err = normed(f, f.abs(), 0, block.norm_attn)
    res = 0.75 * x.double()
    inside(got["x1"], res + n, err + 4 * B.U * (res.abs() + n.abs()) + HALF * (res + n).abs() + 1e-38, "x1")

    # the norm in front of the experts, in 8 bits, as in the test of oled_norm_in
    x1 = got["x1"].double()
    v = x1 / torch.sqrt(x1.pow(2).mean(1, keepdim=True) + EPS) * block.norm_in.double().cpu()
    rel = ((H + 4) / 2 + 8) * B.U
    s = B.row_scales(v)
    inside(got["q_scale"], s, (rel + 4 * B.U) * s, "scales")
    q, u = got["q"].view(B.F8), v / B.spread(s, H)
    inside(q, u, B.f8_step(u * (1 + 1e-4)) / 2 + (2 * rel + 8 * B.U) * u.abs(), "8-bit rows")

    # the gate's logits and the routes
    ref, bound = product(q, got["q_scale"], block.w_gate)
    inside(got["logits"], ref, bound, "logits")
    bias, r = block.bias.cpu(), block.router
    idx, weights, c, val = B.route(got["logits"], bias, mask, E, k, 4, 2, 2, False, True, 2.5)
    near = B.undecided(c, val, k, 4, 2, 2, True, 4e-6 * c.abs().max())
    assert near.float().mean() < 0.1
    ids = got["topk_idx"]
    assert torch.equal(ids[~near], idx[~near].int())
    spread = float(got["logits"].float().max() - got["logits"].float().min())
    sure = (got["weights"].double() - weights).abs() <= (64 + E + 2 * spread) * B.U * weights + 1e-37
    assert sure[~near].all()
    if T >= 33:    # the bias matters here
        plain = B.route(got["logits"], torch.zeros(E), mask, E, k, 4, 2, 2, False, True, 2.5)[0]
        assert not torch.equal(plain, idx)
    counts, offsets, perm, inv = B.permutation(ids, E)
    assert block.counts.tolist() == counts and block.offsets.tolist() == offsets
    assert block.perm[: T * k].tolist() == perm and block.inv_perm[: T * k].tolist() == inv

    # the experts
    raw = T8.unpack(block) if w is T8.SMALL else unpack(block, w)
    table = block.slot_of.tolist() if block.slot_of is not None else range(E)
    o, bound = B.experts(q, got["q_scale"], offsets, perm, k, [raw[b] for b in table])
    R = offsets[-1]
    routed = block.routed[:R].cpu()
    inside(routed, o[:R], bound[:R] + HALF * o[:R].abs() + 1e-37, "experts")
    assert float((routed.double() - o[:R]).norm() / o[:R].norm()) < 2e-2

    # their sum, its norm and gate, onto the residual
    rows = torch.tensor(inv).view(T, k)
    parts = torch.where(rows[:, :, None] < 0, 0.0, routed.double()[rows.clamp_min(0)]) * got["weights"].double()[:, :, None]
    f, mag = parts.sum(1), parts.abs().sum(1)
    n, err = normed(f, mag, k, block.norm_out)
    gt = gate.double()[torch.arange(T) // 32]
    res = 0.75 * x1
    ref = res + n * gt
    inside(y.cpu(), ref, err * gt.abs() + 4 * B.U * (res.abs() + (n * gt).abs()) + HALF * ref.abs() + 1e-38, "y")
    assert torch.equal(y.cpu()[~mask].float(), (0.75 * got["x1"][~mask].float()).bfloat16().float())


def unpack(block, w):
    """As the other test's, for another shape."""
    old = T8.SMALL
    T8.SMALL = w
    try:
        return T8.unpack(block)
    finally:
        T8.SMALL = old
