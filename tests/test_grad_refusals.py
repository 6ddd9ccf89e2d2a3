"""The library computes no gradients: under a gradient mode that would record the call, tensors that require one are refused
rather than left out of the graph without a word.  No GPU: the tensors have no memory, and the library is not reached."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1908_11263_gb300 import qnn
from test_device_refusals import Untouched, prepared

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def new(monkeypatch):
    monkeypatch.setattr(qnn, "_current_device", lambda: 0)
    monkeypatch.setattr(qnn, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(qnn, "_stream", lambda stream: None)
    monkeypatch.setattr(qnn, "_lib", Untouched())
    with FakeTensorMode():
        yield lambda *shape, dtype=BF: torch.empty(shape, dtype=dtype, device="cuda:0")


def calls(new):
    """Name -> a function of the tensor that requires a gradient, and that tensor."""
    x, row = lambda: new(4, 64), lambda: new(64)
    layer, ex = prepared(qnn.PreparedMatmul, 0), prepared(qnn.PreparedExperts, 0, 3)

    def plan():
        return qnn.ExpertPlan(4, 2, 3, torch.device("cuda:0"))

    w32 = lambda *s: new(*s, dtype=F32)
    codes = lambda *s: new(*s, dtype=torch.uint8)
    return {
        "norm x": (lambda t: qnn.block_norm(t), x()),
        "norm residual": (lambda t: qnn.block_norm(x(), t), x()),
        "norm weight": (lambda t: qnn.block_norm(x(), pre_weight=t), row()),
        "norm gate": (lambda t: qnn.block_norm(x(), gate=t), row()),
        "norm out": (lambda t: qnn.block_norm(x(), out=t), x()),
        "logits": (lambda t: qnn.route_topk(t, 2), x()),
        "route bias": (lambda t: qnn.route_topk(x(), 2, bias=t), w32(64)),
        "weights": (lambda t: qnn.PreparedMatmul(t), new(32, 64)),
        "experts' weights": (lambda t: qnn.PreparedExperts(t), new(3, 32, 64)),
        "scale": (lambda t: qnn.PreparedMatmul(codes(32, 64), scale=t, bits=8), w32(32)),
        "bias": (lambda t: qnn.PreparedMatmul(new(32, 64), bias=t), w32(32)),
        "product x": (lambda t: layer(t), x()),
        "product residual": (lambda t: layer(x(), t), new(4, 32)),
        "dispatch x": (lambda t: ex.dispatch(t, plan()), x()),
        "combine x": (lambda t: ex.combine(t, plan(), w32(4, 2)), new(8, 64)),
        "combine weights": (lambda t: ex.combine(new(8, 64), plan(), t), w32(4, 2)),
        "combine residual": (lambda t: ex.combine(new(8, 64), plan(), w32(4, 2), t), new(4, 32)),
    }


NAMES = ["norm x", "norm residual", "norm weight", "norm gate", "norm out", "logits", "route bias", "weights", "experts' weights",
         "scale", "bias", "product x", "product residual", "dispatch x", "combine x", "combine weights", "combine residual"]


@pytest.mark.parametrize("name", NAMES)
def test_refused_where_the_call_would_be_recorded(new, name):
    every = calls(new)
    assert sorted(every) == sorted(NAMES)
    call, t = every[name]
    t.requires_grad_(True)
    with pytest.raises(ValueError, match="gradient"):
        call(t)


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("name", NAMES)
def test_taken_where_it_would_not(new, name, mode):
    call, t = calls(new)[name]
    t.requires_grad_(True)
    with mode(), pytest.raises(AssertionError, match="was reached"):
        call(t)
