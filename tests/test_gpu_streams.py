"""stream= on another stream than the current one: what a call allocates is the launching stream's, so memory that queued
work of the current stream still uses is not handed to it, and temporaries that were laid out may be dropped at once.

Each test holds one stream back with a timed kernel (some twenty milliseconds) and queues on the other."""
import pytest
import torch

from block_util import gen, weights
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
WAIT = 40_000_000  # SM cycles


def outputs(v):
    if isinstance(v, qnn.ExpertPlan):
        return [v._buffer]
    if isinstance(v, (qnn.PreparedMatmul, qnn.PreparedExperts)):
        return [v.image]
    if isinstance(v, qnn.PreparedConv):
        return [v.workspace]
    return [o for o in (v if isinstance(v, tuple) else (v,)) if o is not None]


def results(v):
    """What a call gave, to be compared: a prepared convolution's image has gaps that nothing writes, so it is run."""
    if isinstance(v, qnn.PreparedConv):
        return [v(torch.arange(4 * 16 * 16 * 32, device="cuda").remainder(251).to(torch.uint8).view(4, 16, 16, 32))]
    return outputs(v)


def calls():
    g = gen(1)
    x = torch.randn(64, 512, generator=g, device="cuda").to(BF)
    w, scale, _ = weights(520, 512, 4, BF, g)
    we, se, _ = weights(520, 512, 4, BF, g, 8)
    logits = torch.randn(5000, 64, generator=g, device="cuda")
    ids = torch.randint(0, 8, (64, 2), generator=g, device="cuda", dtype=torch.int32)
    many = torch.randint(0, 8, (5000, 2), generator=g, device="cuda", dtype=torch.int32)
    cw = torch.rand(64, 2, generator=g, device="cuda")
    layer, ex = qnn.PreparedMatmul(w, scale=scale, bits=4), qnn.PreparedExperts(we, scale=se, bits=4)
    plan = qnn.expert_plan(ids, 8)
    h = torch.randn(128, 512, generator=g, device="cuda").to(BF)
    ax = torch.randint(0, 256, (4, 16, 16, 32), generator=g, device="cuda", dtype=torch.uint8)
    cwt = torch.randint(-128, 128, (64, 3, 3, 32), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    kappa = torch.randint(1, 400, (64,), generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    lam = torch.randint(0, 1 << 20, (64,), generator=g, device="cuda", dtype=torch.int32)
    thr = torch.arange(15, device="cuda", dtype=torch.int32).repeat(64, 1) * 1000
    bthr = torch.zeros(64, device="cuda", dtype=torch.int32)
    w4, wb, w8 = cwt[..., :16].contiguous(), cwt[..., :4].contiguous().view(torch.uint8), cwt.view(64, -1)
    a4, ab = ax[..., :16].contiguous(), ax[..., :4].contiguous()
    flat, kw = ax.view(4, -1)[:, :288].contiguous(), dict(shift=16, pad=1)
    pc = qnn.PreparedConv(cwt, kappa, lam, n=4, h=16, wd=16, **kw)
    return {
        "block_norm": lambda s: qnn.block_norm(x, x, stream=s),
        "route_topk": lambda s: qnn.route_topk(logits, 8, stream=s),
        "expert_plan": lambda s: qnn.expert_plan(many, 8, stream=s),
        "matmul": lambda s: layer(x, stream=s),
        "dispatch": lambda s: ex.dispatch(x, plan, stream=s),
        "combine": lambda s: ex.combine(h, plan, cw, stream=s),
        "prepare": lambda s: qnn.PreparedMatmul(w, scale=scale, bits=4, stream=s),
        "prepare_experts": lambda s: qnn.PreparedExperts(we, scale=se, bits=4, stream=s),
        "conv_hwc": lambda s: qnn.conv_hwc(ax, cwt, kappa, lam, stream=s, **kw),
        "conv_hwc_general": lambda s: qnn.conv_hwc(ax, cwt, kappa, lam, stream=s, algo=qnn.ALGO_TC_GENERAL, **kw),
        "conv_hwc_pool2": lambda s: qnn.conv_hwc_pool2(ax, cwt, kappa, lam, stream=s, **kw),
        "conv_hwc_thresholds": lambda s: qnn.conv_hwc_thresholds(a4, w4, thr, bits=4, pad=1, stream=s),
        "conv_binary": lambda s: qnn.conv_binary(ab, wb, bthr, pad=1, stream=s),
        "prepare_conv": lambda s: qnn.PreparedConv(cwt, kappa, lam, n=4, h=16, wd=16, stream=s, **kw),
        "conv_run": lambda s: pc(ax, stream=s),
        "conv_run_pool2": lambda s: pc.pool2(ax, stream=s),
        "linear": lambda s: qnn.linear(flat, w8, stream=s),
        "maxpool": lambda s: qnn.maxpool(ax, stream=s),
        "pack_subbyte": lambda s: qnn.pack_subbyte(cwt, 4, stream=s),
        "unpack_subbyte": lambda s: qnn.unpack_subbyte(ax, 4, False, stream=s),
    }


NAMES = ["block_norm", "route_topk", "expert_plan", "matmul", "dispatch", "combine", "prepare", "prepare_experts", "conv_hwc",
         "conv_hwc_general", "conv_hwc_pool2", "conv_hwc_thresholds", "conv_binary", "prepare_conv", "conv_run", "conv_run_pool2",
         "linear", "maxpool", "pack_subbyte", "unpack_subbyte"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(name):
    every = calls()
    assert sorted(every) == sorted(NAMES)
    call = every[name]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = [o.clone() for o in results(call(None))]
    sizes = [o.untyped_storage().nbytes() for o in outputs(call(side))]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    read = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    held = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    torch.cuda._sleep(WAIT)
    for r, h in zip(read, held):
        r.copy_(h)
    h = None
    held.clear()  # back to the allocator, as memory of the current stream, whose copies are still to come
    got = call(side)
    torch.cuda.synchronize()
    assert all(bool((r == 3).all()) for r in read), "the call wrote to memory that the current stream was still reading"
    assert all(torch.equal(a, b) for a, b in zip(results(got), want))


@pytest.mark.parametrize("experts", [None, 8])
def test_weights_dropped_after_they_were_laid_out(experts):
    g = gen(2)
    w, scale, _ = weights(520, 512, 8, BF, g, experts)
    kind = qnn.PreparedExperts if experts else qnn.PreparedMatmul
    bias = torch.randn(scale.shape, generator=g, device="cuda")
    want = kind(w, scale=scale, bias=bias, bits=8).image.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    args = [v.clone() for v in (w, scale, bias)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
    layer = kind(args[0], scale=args[1], bias=args[2], bits=8, stream=side)
    sizes = [v.untyped_storage().nbytes() for v in args]
    args.clear()
    junk = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes]  # the current stream's next allocations
    torch.cuda.synchronize()
    assert torch.equal(layer.image, want) and all(bool((j == 7).all()) for j in junk)


def test_outputs_dropped_while_the_current_stream_reads_them():
    """The output goes back to the allocator while the current stream still reads it; the next call may not get it."""
    g = gen(3)
    w, scale, _ = weights(520, 512, 8, BF, g)
    layer = qnn.PreparedMatmul(w, scale=scale, bits=8)
    xs = [torch.randn(64, 512, generator=g, device="cuda").to(BF) for _ in range(2)]
    want = layer(xs[0])
    side, read = torch.cuda.Stream(), torch.empty_like(want)
    torch.cuda.synchronize()
    y = layer(xs[0], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(WAIT)
    read.copy_(y)
    y = None
    other = layer(xs[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(read, want) and torch.equal(other, layer(xs[1]))


def test_calls_on_another_stream_can_be_captured():
    g = gen(4)
    w, scale, _ = weights(96, 128, 4, BF, g, 8)
    layer = qnn.PreparedExperts(w, scale=scale, bits=4, dtype=BF)
    ids = torch.randint(0, 8, (40, 2), generator=g, device="cuda", dtype=torch.int32)
    cw = torch.rand(40, 2, generator=g, device="cuda")
    h = torch.randn(80, 128, generator=g, device="cuda").to(BF)
    want = layer.combine(h, qnn.expert_plan(ids, 8), cw)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = layer.combine(h, qnn.expert_plan(ids, 8, stream=side), cw, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        got.zero_()
        graph.replay()
        assert torch.equal(got, want)
