"""qnn.PreparedMatmul and qnn.PreparedExperts against plain products in 64 bits (block_util.py derives the tolerances),
and, on whole numbers, against the exact result."""
import math

import numpy as np
import pytest
import torch

from block_util import U, check, gen, pack, product64, strided, weights
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def run(t, k, m, bits, dtype=BF, gated=False, act="none", bias=False, residual=False, pad=0, out_dtype=None, seed=0):
    g = gen(seed + t + 3 * k + 7 * m + bits)
    rows = 2 * m if gated else m
    w, scale, w64 = weights(rows, k, bits, dtype, g)
    b = torch.randn(rows, generator=g, device="cuda") if bias else None
    x = strided(torch.randn(t, k, generator=g, device="cuda").to(dtype), pad)
    res = strided(torch.randn(t, m, generator=g, device="cuda").to(dtype), pad) if residual else None
    layer = qnn.PreparedMatmul(w, scale=scale, bias=b, bits=bits, dtype=dtype, gated=gated, act=act)
    full = torch.full((t + 2, m + 3), 7.0, dtype=out_dtype or dtype, device="cuda")
    y = layer(x, residual=res, out=full[1:t + 1, :m])
    edge = full.clone()
    edge[1:t + 1, :m] = 7.0
    assert bool((edge == 7.0).all()), "wrote outside its output"
    if t == 0:
        return
    want, err = product64(x, w64, scale, b, m, gated, act)
    if res is not None:
        want = want + res.double()
        err = err + 2.0 ** -23 * want.abs()
    check(y, want, err, f"{t}x{k}x{m} {bits} bits")
    again = layer(x, residual=res, out_dtype=out_dtype)
    assert torch.equal(again, y), "the same call twice differs"


SIZES = [(0, 64, 32), (1, 8, 1), (1, 64, 32), (1, 4096, 257), (3, 72, 40), (7, 200, 100), (8, 1000, 33), (9, 1024, 512),
         (16, 4104, 64), (17, 128, 129), (32, 64, 256), (33, 520, 200), (64, 2048, 384), (100, 1096, 1001), (129, 64, 300),
         (257, 512, 513), (300, 4096, 128), (513, 200, 700), (1100, 1024, 264)]


@pytest.mark.parametrize("t,k,m", SIZES)
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_sizes(t, k, m, bits, dtype):
    run(t, k, m, bits, dtype)


@pytest.mark.parametrize("t,k,m", [(1, 512, 8), (5, 264, 17), (16, 1024, 100), (40, 136, 72), (200, 648, 130), (700, 256, 520)])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
def test_gated(t, k, m, bits, act):
    run(t, k, m, bits, BF if bits % 8 else HF, gated=True, act=act, bias=True, residual=bits == 4)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("t", [4, 50, 400])
@pytest.mark.parametrize("bias,residual", [(True, False), (False, True), (True, True)])
def test_epilogue(act, t, bias, residual):
    run(t, 320, 136, 8, BF, act=act, bias=bias, residual=residual)


@pytest.mark.parametrize("pad", [1, 2, 5, 8, 24])
@pytest.mark.parametrize("t", [2, 24, 300])
def test_strides(pad, t):
    run(t, 328, 200, 4, HF, residual=True, pad=pad)
    run(t, 77, 200, 16, BF, residual=True, pad=pad)   # odd rows


@pytest.mark.parametrize("t", [1, 12, 90, 520])
def test_float_outputs(t):
    run(t, 1024, 300, 8, HF, out_dtype=F32, bias=True)
    run(t, 1024, 300, 16, BF, out_dtype=F32, gated=True, act="silu")


@pytest.mark.parametrize("t", [1, 8, 31, 70, 400])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_whole_numbers_are_exact(t, bits, dtype):
    """Whole-numbered x and codes with sums below 2^24: every partial sum is exact, so the result is."""
    k, m, g = 2056, 200, gen(t + bits)
    x = torch.randint(-8, 9, (t, k), generator=g, device="cuda")
    lo, hi = (-128, 128) if bits == 16 else (-(1 << (bits - 1)), 1 << (bits - 1))
    codes = torch.randint(lo, hi, (m, k), generator=g, device="cuda")
    codes[0], codes[1] = lo, hi - 1
    w = codes.to(dtype) if bits == 16 else pack(codes, bits)
    y = qnn.PreparedMatmul(w, bits=bits, dtype=dtype)(x.to(dtype), out_dtype=F32)
    assert torch.equal(y.double(), x.double() @ codes.double().t())


@pytest.mark.parametrize("t", [5, 60, 300])
@pytest.mark.parametrize("bits", [16, 4])
def test_nonfinite_rows_stay_alone(t, bits):
    g = gen(9)
    w, scale, _ = weights(100, 136, bits, BF, g)
    layer = qnn.PreparedMatmul(w, scale=scale, bits=bits, dtype=BF)
    x = torch.randn(t, 136, generator=g, device="cuda").to(BF)
    want = layer(x)
    x2 = x.clone()
    x2[2, 7], x2[4, 135] = math.nan, math.inf
    got = layer(x2)
    rest = [i for i in range(t) if i not in (2, 4)]
    assert torch.equal(got[rest], want[rest])
    assert bool(got[2].isnan().all()) and not bool(got[4].isfinite().all())


def test_residual_in_place_and_other_stream():
    g = gen(4)
    w, scale, _ = weights(264, 256, 4, BF, g)
    layer = qnn.PreparedMatmul(w, scale=scale, bits=4, dtype=BF, act="silu")
    for t in (3, 40, 300):
        x = torch.randn(t, 256, generator=g, device="cuda").to(BF)
        res = torch.randn(t, 264, generator=g, device="cuda").to(BF)
        want = layer(x, residual=res)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = layer(x, residual=res)
        s.synchronize()
        got = layer(x, residual=res, out=res)
        assert got is res and torch.equal(got, want) and torch.equal(other, want)


def test_a_graph_replays_it():
    g = gen(5)
    w, scale, _ = weights(520, 512, 8, BF, g)
    layer = qnn.PreparedMatmul(w, scale=scale, bits=8, dtype=BF)
    for t in (4, 300):
        x = torch.randn(t, 512, generator=g, device="cuda").to(BF)
        out = torch.empty(t, 520, dtype=BF, device="cuda")
        layer(x, out=out)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            layer(x, out=out)
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(x, out=out)
        x.copy_(torch.randn(t, 512, generator=g, device="cuda"))
        out.zero_()
        graph.replay()
        assert torch.equal(out, layer(x))


# ---------------------------------------------------------------- experts

def routed(t, top, experts, g, dropped=0.0, crowd=None):
    ids = torch.rand(t, experts, generator=g, device="cuda").topk(top, -1).indices.int() if t else \
        torch.empty(0, top, dtype=torch.int32, device="cuda")
    if crowd is not None and t:
        ids[:, 0] = crowd
        if top > 1:
            ids[:, 1:] = torch.where(ids[:, 1:] == crowd, (crowd + 1) % experts, ids[:, 1:])
    if dropped:
        ids[torch.rand(t, top, generator=g, device="cuda") < dropped] = -1
    w = torch.rand(t, top, generator=g, device="cuda")
    return ids, w


EXPERTS = [(0, 2, 4, 64, 32), (1, 1, 1, 8, 1), (1, 4, 16, 256, 72), (5, 2, 8, 200, 100), (16, 4, 64, 512, 96),
           (70, 3, 5, 136, 257), (300, 2, 4, 264, 200), (900, 6, 16, 128, 130)]


@pytest.mark.parametrize("t,top,experts,k,m", EXPERTS)
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("gated", [False, True])
def test_dispatch(t, top, experts, k, m, bits, gated):
    dtype = HF if bits in (8, 2) else BF
    g = gen(t + bits + k)
    rows = 2 * m if gated else m
    w, scale, w64 = weights(rows, k, bits, dtype, g, experts)
    b = torch.randn(experts, rows, generator=g, device="cuda")
    ids, _ = routed(t, top, experts, g, dropped=0.2 if t > 4 else 0.0, crowd=1 if t == 300 else None)
    x = strided(torch.randn(t, k, generator=g, device="cuda").to(dtype), 3 if t == 70 else 0)
    plan = qnn.expert_plan(ids, experts)
    layer = qnn.PreparedExperts(w, scale=scale, bias=b, bits=bits, dtype=dtype, gated=gated, act="silu")
    full = torch.full((t * top + 2, m + 1), 7.0, dtype=dtype, device="cuda")
    y = layer.dispatch(x, plan, out=full[1:-1, :m])
    edge = full.clone()
    edge[1:-1, :m] = 7.0
    assert bool((edge == 7.0).all()), "wrote outside its output"
    off, order = plan.offsets.tolist(), plan.order.tolist()
    for e in range(experts):
        if off[e] == off[e + 1]:
            continue
        at = torch.tensor([order[p] // top for p in range(off[e], off[e + 1])], device="cuda")
        want, err = product64(x[at], w64[e], None if scale is None else scale[e], b[e], m, gated, "silu")
        check(y[off[e]:off[e + 1]], want, err, f"expert {e}")
    assert bool((y[off[-1]:] == 0).all())
    assert torch.equal(layer.dispatch(x, plan), y)


@pytest.mark.parametrize("t,top,experts,k,m", EXPERTS)
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
@pytest.mark.parametrize("residual", [False, True])
def test_combine(t, top, experts, k, m, bits, residual):
    dtype = BF if bits in (8, 2) else HF
    g = gen(t + bits + k + 1)
    w, scale, w64 = weights(m, k, bits, dtype, g, experts)
    b = torch.randn(experts, m, generator=g, device="cuda")
    ids, cw = routed(t, top, experts, g, dropped=0.2 if t > 4 else 0.0, crowd=0 if t == 900 else None)
    if t > 4:
        ids[3] = -1                    # a token that no expert serves
        cw[ids < 0] = math.nan         # weights of left-out choices count for nothing
    plan = qnn.expert_plan(ids, experts)
    h = torch.randn(t * top, k, generator=g, device="cuda").to(dtype)
    off = plan.offsets.tolist()
    h[off[-1]:] = math.nan             # rows after the last place are not read
    res = torch.randn(t, m, generator=g, device="cuda").to(dtype) if residual else None
    layer = qnn.PreparedExperts(w, scale=scale, bias=b, bits=bits, dtype=dtype)
    y = layer.combine(h, plan, cw, residual=res)
    assert y.shape == (t, m) and y.dtype == dtype
    if t == 0:
        return
    want = torch.zeros(t, m, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(want)
    order = plan.order.long()
    for e in range(experts):
        if off[e] == off[e + 1]:
            continue
        slots = order[off[e]:off[e + 1]]
        v, ev = product64(h[off[e]:off[e + 1]], w64[e], None if scale is None else scale[e], b[e], m, False, "none")
        f = cw.reshape(-1)[slots].double()[:, None]
        want.index_add_(0, slots // top, f * v)
        err.index_add_(0, slots // top, f * (ev + (top + 1) * 2.0 ** -24 * v.abs()))
    if res is not None:
        want, err = want + res.double(), err + 2.0 ** -23 * (want.abs() + res.double().abs())
    check(y, want, err)
    if t > 4:
        assert torch.equal(y[3], res[3] if residual else torch.zeros_like(y[3]))
    assert torch.equal(layer.combine(h, plan, cw, residual=res), y)


def test_a_graph_keeps_its_own_workspace():
    """A captured combine replays correctly after later calls have outgrown the stream's shared workspace."""
    g = gen(11)
    w, scale, _ = weights(96, 128, 4, BF, g, 8)
    layer = qnn.PreparedExperts(w, scale=scale, bits=4, dtype=BF)
    ids, cw = routed(40, 2, 8, g)
    plan = qnn.expert_plan(ids, 8)
    h = torch.randn(80, 128, generator=g, device="cuda").to(BF)
    out = torch.empty(40, 96, dtype=BF, device="cuda")
    want = layer.combine(h, plan, cw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.combine(h, plan, cw, out=out)
    big_ids, big_w = routed(4000, 2, 8, g)
    big = qnn.expert_plan(big_ids, 8)
    layer.combine(torch.randn(8000, 128, generator=g, device="cuda").to(BF), big, big_w)
    torch.cuda.empty_cache()
    junk = [torch.full((1 << 18,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all(bool((j == 7).all()) for j in junk)


# ---------------------------------------------------------------- refusals

def test_refusals():
    w = torch.zeros(32, 64, device="cuda", dtype=BF)
    layer = qnn.PreparedMatmul(w)
    x = torch.zeros(4, 64, device="cuda", dtype=BF)
    for bad, error in ((x[:, :63], ValueError), (x.half(), TypeError), (x.cpu(), ValueError), (x[0], ValueError),
                       (torch.zeros(4, 128, device="cuda", dtype=BF)[:, ::2], ValueError)):
        with pytest.raises(error):
            layer(bad)
    with pytest.raises(ValueError):
        layer(x, residual=torch.zeros(4, 31, device="cuda", dtype=BF))
    with pytest.raises(TypeError):
        layer(x, residual=torch.zeros(4, 32, device="cuda"))
    with pytest.raises(TypeError):
        layer(x, out=torch.zeros(4, 32, device="cuda", dtype=HF))
    with pytest.raises(TypeError):
        layer(x, out_dtype=torch.float64)
    codes = torch.zeros(32, 16, device="cuda", dtype=torch.uint8)
    for kw, error in ((dict(bits=3), qnn.QnnError), (dict(bits=4, dtype=F32), TypeError), (dict(bits=4, act="tanh"), ValueError),
                      (dict(bits=4, scale=torch.ones(31, device="cuda")), ValueError), (dict(bits=16), TypeError),
                      (dict(bits=4, scale=torch.ones(32, device="cuda", dtype=HF)), TypeError)):
        with pytest.raises(error):
            qnn.PreparedMatmul(codes, **kw)
    with pytest.raises(ValueError):
        qnn.PreparedMatmul(codes[:31], bits=4, gated=True)
    with pytest.raises(ValueError):
        qnn.PreparedExperts(codes, bits=4)
    ex = qnn.PreparedExperts(torch.zeros(4, 8, 64, device="cuda", dtype=BF))
    plan = qnn.expert_plan(torch.zeros(4, 2, device="cuda", dtype=torch.int32), 4)
    other = qnn.expert_plan(torch.zeros(4, 2, device="cuda", dtype=torch.int32), 5)
    with pytest.raises(ValueError):
        ex.dispatch(x, other)
    with pytest.raises(ValueError):
        ex.dispatch(x[:3], plan)
    with pytest.raises(ValueError):
        ex.combine(x, plan, torch.zeros(4, 2, device="cuda"))       # a row per place is needed
    with pytest.raises(TypeError):
        ex.combine(x.repeat(2, 1), plan, torch.zeros(4, 2, device="cuda", dtype=HF))
    with pytest.raises(ValueError):
        ex.combine(x.repeat(2, 1), plan, None)
