"""Host threads that call the library at once on one stream.  ctypes lets go of the interpreter lock during a foreign call,
and torch gives every thread the same current stream, so the launches of two calls interleave: what a call keeps between
its launches must be its own.  Two calls that are inside the library at the same time have to hold different workspaces;
and whole runs of calls are compared with the results of the same calls made alone, bit by bit (the kernels add in a fixed
order)."""
import ctypes
import sys
import threading

import pytest
import torch

from block_util import gen, weights
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def at_once(calls, rounds):
    """Runs each of `calls` `rounds` times in a thread of its own; returns the outputs by call."""
    got = [[] for _ in calls]
    errors = []
    start = threading.Barrier(len(calls))

    def work(i):
        try:
            start.wait(30)
            for _ in range(rounds):
                got[i].append(calls[i]())
        except Exception as e:  # reported by the test's own thread
            errors.append(e)

    old = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(old)
    assert not errors, errors
    torch.cuda.synchronize()
    return got


def check(calls, rounds=400):
    want = [c() for c in calls]
    torch.cuda.synchronize()
    for i, outs in enumerate(at_once(calls, rounds)):
        bad = sum(not all(torch.equal(a, b) for a, b in zip(o, want[i])) for o in outs)
        assert bad == 0, f"call {i}: {bad} of {rounds} results differ from the same call made alone"


def experts_layer(t, top, experts, k, m, seed):
    g = gen(seed)
    w, scale, _ = weights(m, k, 4, BF, g, experts)
    layer = qnn.PreparedExperts(w, scale=scale, bits=4, dtype=BF)
    ids = torch.rand(t, experts, generator=g, device="cuda").topk(top, -1).indices.int()
    cw = torch.rand(t, top, generator=g, device="cuda")
    return layer, ids, cw, g


class Meeting:
    """The library, but for one function: a call of it that has its workspace waits inside until a second one is there too,
    and returns without running.  `held` are the workspaces that the calls had."""

    def __init__(self, lib, name, place):
        self._lib, self._name, self._place, self.held = lib, name, place, []
        self._both = threading.Barrier(2)

    def __getattr__(self, name):
        real = getattr(self._lib, name)
        return self._enter if name == self._name else real

    def _enter(self, *args):
        ws = args[self._place]
        ws = ws.value if isinstance(ws, ctypes.c_void_p) else ws
        if not ws:
            return qnn.QNN_EWORKSPACE
        self.held.append(ws)
        self._both.wait(30)
        return qnn.QNN_OK


def conv_layer(g):
    x = torch.randint(0, 256, (2, 8, 8, 32), generator=g, device="cuda", dtype=torch.uint8)
    w = torch.randint(-128, 128, (64, 3, 3, 32), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    kappa = torch.randint(1, 400, (64,), generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    lam = torch.randint(0, 1 << 20, (64,), generator=g, device="cuda", dtype=torch.int32)
    return x, w, kappa, lam


@pytest.mark.parametrize("name,place", [("qnn_experts_combine", 14), ("qnn_experts_dispatch", 11), ("qnn_matmul_run", 11),
                                        ("qnn_expert_plan", 6), ("qconv_hwc", 8)])
def test_calls_at_once_hold_different_workspaces(monkeypatch, name, place):
    layer, ids, cw, g = experts_layer(200, 2, 4, 136, 96, 7)
    plan = qnn.expert_plan(ids, 4)
    x = torch.randn(400, 137, generator=g, device="cuda").to(BF)[:, :136]
    w, scale, _ = weights(96, 136, 8, BF, g)
    product = qnn.PreparedMatmul(w, scale=scale, bits=8, dtype=BF)
    many = torch.randint(0, 16, (3000, 4), generator=g, device="cuda", dtype=torch.int32)
    conv = conv_layer(g)
    call = {"qnn_experts_combine": lambda: layer.combine(x, plan, cw), "qnn_experts_dispatch": lambda: layer.dispatch(x[:200], plan),
            "qnn_matmul_run": lambda: product(x), "qnn_expert_plan": lambda: qnn.expert_plan(many, 16),
            "qconv_hwc": lambda: qnn.conv_hwc(*conv, shift=16, pad=1, algo=qnn.ALGO_TC_GENERAL)}[name]
    call()
    lib = Meeting(qnn.load(), name, place)
    monkeypatch.setattr(qnn, "_lib", lib)
    at_once([call, call], 1)
    assert len(lib.held) == 2 and lib.held[0] != lib.held[1]


@pytest.mark.parametrize("t", [24, 200])  # streamed products; the tensor cores
def test_combine(t):
    layer, ids, cw, g = experts_layer(t, 2, 4, 136, 96, t)
    plan = qnn.expert_plan(ids, 4)
    hs = [torch.randn(2 * t, 137, generator=g, device="cuda").to(BF)[:, :136] for _ in range(2)]  # rows copied first
    check([lambda h=h: (layer.combine(h, plan, cw),) for h in hs])


def test_dispatch():
    layer, ids, _, g = experts_layer(200, 2, 4, 136, 96, 3)
    plan = qnn.expert_plan(ids, 4)
    xs = [torch.randn(200, 136, generator=g, device="cuda").to(BF) for _ in range(2)]
    check([lambda x=x: (layer.dispatch(x, plan),) for x in xs])


def test_product_of_unaligned_rows():
    g = gen(4)
    w, scale, _ = weights(96, 136, 8, BF, g)
    layer = qnn.PreparedMatmul(w, scale=scale, bits=8, dtype=BF)
    xs = [torch.randn(300, 137, generator=g, device="cuda").to(BF)[:, :136] for _ in range(2)]
    check([lambda x=x: (layer(x),) for x in xs])


def test_plans():
    def parts(ids):
        p = qnn.expert_plan(ids, 16)
        return p.offsets, p.order, p.position

    g = gen(5)
    ids = [torch.randint(0, 16, (3000 + 500 * i, 4), generator=g, device="cuda", dtype=torch.int32) for i in range(2)]
    check([lambda v=v: parts(v) for v in ids])


def test_convolutions():
    layers = [conv_layer(gen(6 + i)) for i in range(2)]
    check([lambda v=v: (qnn.conv_hwc(*v, shift=16, pad=1, algo=qnn.ALGO_TC_GENERAL),) for v in layers])
