"""Tensors and streams of another device than the current one are refused before the library is reached, which launches on
the current device and asks it for its properties.  No GPU: the tensors have no memory, and the device query is replaced."""
import types

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_1908_11263_gb300 import qnn

BF, U8, I8, I16, I32 = torch.bfloat16, torch.uint8, torch.int8, torch.int16, torch.int32


class Untouched:
    def __getattr__(self, name):
        if name.endswith("_size"):  # host arithmetic
            return lambda *a: qnn.QNN_OK

        def reached(*a):
            raise AssertionError(f"{name} was reached")

        return reached


@pytest.fixture
def device(monkeypatch):
    """cuda:0 is current; returns what makes tensors."""
    monkeypatch.setattr(qnn, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(device=torch.device("cuda:0"), cuda_stream=0))
    monkeypatch.setattr(qnn, "_lib", Untouched())
    with FakeTensorMode():
        yield lambda *shape, dtype=BF, at=1: torch.empty(shape, dtype=dtype, device=f"cuda:{at}")


def prepared(kind, at, experts=1):
    layer = object.__new__(kind)
    layer.dtype, layer.device, layer.experts, layer.m, layer.k = BF, torch.device(f"cuda:{at}"), experts, 32, 64
    layer.nbytes, layer._desc, layer._image = 0, None, 0
    return layer


def prepared_conv():
    layer = object.__new__(qnn.PreparedConv)
    layer.desc, layer.out_shape, layer.oh, layer.ow, layer.nbytes, layer.workspace = qnn.ConvDesc(), (1, 8, 8, 32), 8, 8, 0, None
    return layer


def calls(t, at, stream=None):
    """Every entry point with tensors on cuda:`at`."""
    def new(*shape, dtype=BF):
        return t(*shape, dtype=dtype, at=at)

    def plan():
        p = qnn.ExpertPlan(4, 2, 3, torch.device(f"cuda:{at}"))
        return p

    x, act, w = lambda: new(4, 64), lambda: new(1, 8, 8, 32, dtype=U8), lambda: new(32, 3, 3, 32, dtype=I8)
    kappa, lam = lambda: new(32, dtype=I16), lambda: new(32, dtype=I32)
    return {
        "block_norm": lambda: qnn.block_norm(x(), stream=stream),
        "route_topk": lambda: qnn.route_topk(x(), 2, stream=stream),
        "expert_plan": lambda: qnn.expert_plan(new(4, 2, dtype=I32), 3, stream=stream),
        "PreparedMatmul": lambda: qnn.PreparedMatmul(new(32, 64), stream=stream),
        "PreparedExperts": lambda: qnn.PreparedExperts(new(3, 32, 64), stream=stream),
        "matmul": lambda: prepared(qnn.PreparedMatmul, at)(x(), stream=stream),
        "dispatch": lambda: prepared(qnn.PreparedExperts, at, 3).dispatch(x(), plan(), stream=stream),
        "combine": lambda: prepared(qnn.PreparedExperts, at, 3).combine(new(8, 64), plan(), new(4, 2, dtype=torch.float32), stream=stream),
        "conv_hwc": lambda: qnn.conv_hwc(act(), w(), kappa(), lam(), pad=1, stream=stream),
        "conv_hwc_pool2": lambda: qnn.conv_hwc_pool2(act(), w(), kappa(), lam(), pad=1, stream=stream),
        "conv_hwc_thresholds": lambda: qnn.conv_hwc_thresholds(new(1, 8, 8, 16, dtype=U8), new(32, 3, 3, 16, dtype=I8),
                                                               new(32, 15, dtype=I32), bits=4, pad=1, stream=stream),
        "conv_binary": lambda: qnn.conv_binary(new(1, 8, 8, 4, dtype=U8), new(32, 3, 3, 4, dtype=U8), lam(), pad=1, stream=stream),
        "conv_hwc_noalloc": lambda: qnn.conv_hwc_noalloc(act(), w(), kappa(), lam(), act(), pad=1, stream=stream),
        "PreparedConv": lambda: qnn.PreparedConv(w(), kappa(), lam(), n=1, h=8, wd=8, pad=1, stream=stream),
        "conv_run": lambda: prepared_conv()(act(), stream=stream),
        "conv_run_pool2": lambda: prepared_conv().pool2(act(), stream=stream),
        "linear": lambda: qnn.linear(new(4, 64, dtype=U8), new(32, 64, dtype=I8), stream=stream),
        "maxpool": lambda: qnn.maxpool(act(), stream=stream),
        "pack_subbyte": lambda: qnn.pack_subbyte(w(), 4, stream=stream),
        "unpack_subbyte": lambda: qnn.unpack_subbyte(act(), 4, False, stream=stream),
    }


NAMES = ["block_norm", "route_topk", "expert_plan", "PreparedMatmul", "PreparedExperts", "matmul", "dispatch", "combine", "conv_hwc",
         "conv_hwc_pool2", "conv_hwc_thresholds", "conv_binary", "conv_hwc_noalloc", "PreparedConv", "conv_run", "conv_run_pool2",
         "linear", "maxpool", "pack_subbyte", "unpack_subbyte"]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device(device, name):
    every = calls(device, 1)
    assert sorted(every) == sorted(NAMES)
    with pytest.raises(ValueError, match="current device"):
        every[name]()


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device(device, name):
    stream = types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=5)
    with pytest.raises(ValueError, match="current device"):
        calls(device, 0, stream)[name]()


def test_streams_without_tensors(device):
    stream = types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=5)
    for call in (lambda: qnn.device_status(stream), lambda: qnn.selftest_wait_timeout(1000, stream)):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.parametrize("name", ["block_norm", "route_topk", "matmul", "linear"])
def test_tensors_of_the_current_device_pass(device, monkeypatch, name):
    """The same calls with everything on the current device get as far as the library."""
    monkeypatch.setattr(qnn, "_raw_stream", lambda index: 0)
    with pytest.raises(AssertionError, match="was reached"):
        calls(device, 0)[name]()


def test_outputs_and_constants_elsewhere(device):
    """What the library writes to, and what only some calls have, is looked at as well."""
    def there(*shape, dtype=U8):
        return torch.empty(shape, dtype=dtype, device="cuda:1")

    def here(*shape, dtype=U8):
        return device(*shape, dtype=dtype, at=0)

    act, w, kappa, lam = here(1, 8, 8, 32), here(32, 3, 3, 32, dtype=I8), here(32, dtype=I16), here(32, dtype=I32)
    x = here(4, 64, dtype=BF)
    for call in (lambda: qnn.linear(here(4, 64), here(32, 64, dtype=I8), out=there(4, 32, dtype=I32)),
                 lambda: qnn.maxpool(act, out=there(1, 4, 4, 32)), lambda: prepared_conv()(act, out=there(1, 8, 8, 32)),
                 lambda: qnn.pack_subbyte(w, 4, out=there(32, 3, 3, 16)), lambda: qnn.unpack_subbyte(act, 4, True, out=there(1, 8, 8, 64, dtype=I8)),
                 lambda: qnn.PreparedConv(w, kappa, lam, n=1, h=8, wd=8, pad=1, bias=there(32, dtype=I32)),
                 lambda: qnn.conv_hwc(act, w, kappa, lam, pad=1, workspace=there(1 << 20)),
                 lambda: qnn.block_norm(x, out=there(4, 64, dtype=BF)), lambda: qnn.block_norm(x, gate=there(64, dtype=BF)),
                 lambda: qnn.route_topk(x, 2, bias=there(64, dtype=torch.float32)),
                 lambda: prepared(qnn.PreparedMatmul, 0)(x, out=there(4, 32, dtype=BF))):
        with pytest.raises(ValueError):
            call()
