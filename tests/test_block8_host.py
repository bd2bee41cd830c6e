"""The chained block's host side: its library calls replaced by stand-ins on the CPU."""
import contextlib

import pytest
import torch

from paper_2609_33385_amd import block8, oled

H, I, E, K, TOKENS = 256, 128, 16, 4, 64
CALLS = ["oled_norm_in", "oled_fp8_matmul", "oled_norm_out", "oled_norm_in", "oled_fp8_matmul",
         "oled_route_scored", "oled_fp8_experts", "oled_norm_out"]
OUTPUT = {"oled_norm_in": 8, "oled_fp8_matmul": 9, "oled_norm_out": 13, "oled_route_scored": 5,
          "oled_fp8_experts": 12}


class Stage(tuple):
    pass


class Stream:
    """As much of torch.cuda.Stream as the block uses; events are the stream's name."""

    def __init__(self, name, log):
        self.name, self.log, self.cuda_stream = name, log, hash(name) % 1000 + 1

    def record_event(self):
        self.log.append(("record", self.name))
        return self.name

    def wait_event(self, event):
        self.log.append(("wait", self.name, event))


@pytest.fixture
def stage(monkeypatch):
    """(log, fail): the calls made, and the index of one that is refused."""
    log, fail = [], []

    def stand_in(name):
        def call(*args):
            stream, out = args[-1], args[OUTPUT[name]]
            refused = len([c for c in log if c[0] == "call"]) in fail
            log.append(("call", name, stream.name if stream is not None else None))
            if refused:
                return oled.OLED_ERR_UNSUPPORTED
            out.zero_()
            return oled.OLED_OK
        return call
    for name in OUTPUT:
        monkeypatch.setattr(oled, name, stand_in(name))
    made = Stream("made", log)
    capturing = []      # names of streams under capture
    within = []

    @contextlib.contextmanager
    def on(stream):
        within.append(stream.name)
        yield
        within.pop()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: made)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: within[-1] in capturing)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("held", s.name, t.data_ptr())))
    log_and_fail = Stage((log, fail))
    log_and_fail.capturing = capturing
    return log_and_fail


def weights(rows, cols):
    nb = -(-rows // 128)
    return torch.zeros((rows, cols), dtype=torch.uint8), torch.ones((nb, cols // 128))


def make(tokens=TOKENS, **kw):
    router = oled.Router(n_experts=E, top_k=K, n_groups=4, top_groups=2, group_best=2, score=1, renorm=1, scale=1.0)
    experts = torch.zeros((E, oled.oled_fp8_expert_bytes(H, I)), dtype=torch.uint8)
    return block8.Block8(router, H, I, tokens, weights(H, H), weights(E, H), experts, **kw)


def rows(T, value=3.0):
    return torch.full((T, H), value, dtype=torch.bfloat16)


def test_calls(stage):
    log, _ = stage
    x = rows(5)
    assert make().forward(x, rows(5), stream=Stream("a", log)) is x
    assert [c[1:] for c in log if c[0] == "call"] == [(n, "a") for n in CALLS]
    assert (x == 0).all()      # the last call's output


@pytest.mark.parametrize("at", range(8))
def test_refused_call_leaves_x(stage, at):
    log, fail = stage
    block = make()
    fail.append(at)
    x = rows(5)
    with pytest.raises(oled.OledError, match=CALLS[at]):
        block.forward(x, rows(5), stream=Stream("a", log))
    assert (x == 3).all()
    assert len([c for c in log if c[0] == "call"]) == at + 1


def test_routing_workspace_serves_fewer_tokens():
    """A block for many tokens routes any fewer: the workspace it keeps is no smaller
    than what each number of tokens asks for."""
    for tokens in (8193, 20000):
        kept = oled.oled_route_scored_workspace(tokens, E)
        assert all(oled.oled_route_scored_workspace(T, E) <= kept for T in (1, 64, 4096, 8191, 8192, tokens))


def order(log):
    """Waits, and where calls run, each run of calls once."""
    out = []
    for c in log:
        c = c[:3] if c[0] == "wait" else (c[0], c[-1]) if c[0] == "call" else None
        if c and (not out or out[-1] != c):
            out.append(c)
    return out


def test_streams_follow_each_other(stage):
    """A call on another stream waits for the stream of the one before (the first: for the
    stream the block was made on); calls on one stream add nothing."""
    log, _ = stage
    a, b = Stream("a", log), Stream("b", log)
    block = make(bias=torch.zeros(E))
    for s in (a, a, b, a, None):
        block.forward(rows(3), rows(3), stream=s)
    assert order(log) == [("wait", "a", "made"), ("call", "a"), ("wait", "b", "a"), ("call", "b"),
                          ("wait", "a", "b"), ("call", "a"), ("wait", "made", "a"), ("call", "made")]
    for name in ("a", "b"):      # every tensor is held for each stream, once
        held = [c[2] for c in log if c[:2] == ("held", name)]
        assert len(held) == len(set(held))
        for t in (*block.w_out, *block.w_gate, block.experts, block.bias, block.norm_in, block.q, block.q_scale,
                  block.f, block.x1, block.logits, block.topk_idx, block.weights, block.counts, block.offsets,
                  block.perm, block.inv_perm, block.routed, block.route_ws, block.expert_ws):
            assert t.data_ptr() in held


def test_no_wait_while_recorded(stage):
    """A stream under capture cannot wait for work outside of it; the next call that is
    not recorded follows the last one that was not."""
    log, _ = stage
    a, b, g = Stream("a", log), Stream("b", log), Stream("g", log)
    stage.capturing.append("g")
    block = make()
    for s in (a, g, a, g, b):
        block.forward(rows(3), rows(3), stream=s)
    assert order(log) == [("wait", "a", "made"), ("call", "a"), ("call", "g"), ("call", "a"), ("call", "g"),
                          ("wait", "b", "a"), ("call", "b")]


F32, I32, U8, BF16 = torch.float32, torch.int32, torch.uint8, torch.bfloat16


@pytest.mark.parametrize("change", [
    dict(token_mask=torch.ones(4, dtype=U8)), dict(token_mask=torch.ones(5, dtype=torch.int64)),
    dict(token_mask=torch.ones(10, dtype=U8)[::2]), dict(gate=torch.ones(H - 1)), dict(gate=torch.ones(H).double()),
    dict(gate=torch.ones((2, H)), gate_tokens=2), dict(gate=torch.ones((H, 2)).t()[0]),
    dict(gate=torch.ones((1, H), dtype=BF16)), dict(gate=torch.ones((4, H)), gate_tokens=1)])
def test_short_or_wrong_call_arguments(stage, change):
    """Refused before any call is made; x is as it was."""
    log, _ = stage
    block, x = make(), rows(5)
    with pytest.raises(ValueError, match="must be contiguous"):
        block.forward(x, rows(5), stream=Stream("a", log), **change)
    assert not log and (x == 3).all()


@pytest.mark.parametrize("change", [
    dict(token_mask=torch.ones(5, dtype=torch.bool)), dict(token_mask=torch.ones(9, dtype=U8)),
    dict(gate=torch.ones(H)), dict(gate=torch.ones((1, H))), dict(gate=torch.ones((3, H)), gate_tokens=2),
    dict(gate=torch.ones((1, H)), gate_tokens=5), dict(gate=torch.ones((1, H)), gate_tokens=500)])
def test_right_call_arguments(stage, change):
    log, _ = stage
    make().forward(rows(5), rows(5), stream=Stream("a", log), **change)
    assert len([c for c in log if c[0] == "call"]) == 8


@pytest.mark.parametrize("change", [
    dict(bias=torch.zeros(E - 1)), dict(bias=torch.zeros(E, dtype=BF16)), dict(slot_of=torch.zeros(E)),
    dict(slot_of=torch.zeros(E - 1, dtype=I32)), dict(norm_in=torch.ones(H - 8)), dict(norm_attn=torch.ones(8)),
    dict(norm_out=torch.ones(H).double()), dict(norm_out=torch.ones(2 * H)[::2]), dict(tokens=0), dict(tokens=65536),
    dict(hidden=200), dict(inter=64), dict(hidden=1 << 15), dict(w_out=weights(128, H)), dict(w_gate=weights(8, H)),
    dict(w_out=(torch.zeros((H, H)), torch.ones((2, 2)))), dict(w_gate=(torch.zeros((E, H), dtype=U8), torch.ones(1))),
    dict(experts=torch.zeros((E, 256), dtype=U8)), dict(experts=torch.zeros(9, dtype=U8)), dict(blocks=E - 1)])
def test_short_or_wrong_parts(stage, change):
    router = oled.Router(n_experts=E, top_k=K, n_groups=4, top_groups=2, group_best=2, score=1, renorm=1, scale=1.0)
    size = oled.oled_fp8_expert_bytes(H, I)
    part = dict(hidden=H, inter=I, tokens=8, w_out=weights(H, H), w_gate=weights(E, H),
                experts=torch.zeros((change.pop("blocks", E), size), dtype=U8))
    part.update(change)
    args = [part.pop(n) for n in ("hidden", "inter", "tokens", "w_out", "w_gate", "experts")]
    with pytest.raises(ValueError, match="must be"):
        block8.Block8(router, *args, **part)
