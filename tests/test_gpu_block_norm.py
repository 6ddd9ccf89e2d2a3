"""qnn.block_norm against a plain implementation in 64 bits.

Tolerance, from the arithmetic: an output is rounded once to its type (unit roundoff U below); before that each value
passes fewer than 100 roundings of 2^-24 (a thread's sum of at most 32 squares, a tree of 10 more, and a few products),
each relative to the largest intermediate of its row: 100 * 2^-24 < 2^-17."""
import math

import pytest
import torch

from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
GUARD = 7.0


def reference(x, residual, gate, post, pw, pb, w, b, scale, eps, kind):
    def norm(v, w, b):
        mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
        f = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
        y = (v - mean) * f
        big = (v.abs() + mean.abs()) * f
        if w is not None:
            y, big = y * w.double(), big * w.double().abs()
        if b is not None:
            y, big = y + b.double(), big + b.double().abs()
        return y, big

    u = x.double()
    big = u.abs()
    if post:
        u, big = norm(u, pw, pb)
    g = torch.ones_like(u)
    if gate is not None:
        rows = gate if gate.dim() == 2 else gate[None]
        g = rows.double().repeat_interleave(x.shape[0] // rows.shape[0], 0)
    r = scale * g * u + (0 if residual is None else residual.double())
    big = (scale * g).abs() * big + (0 if residual is None else residual.double().abs())
    h, bigh = norm(r, w, b)
    f = 1 / torch.sqrt((r * r).mean(1, keepdim=True) + eps) if kind == "rms" else \
        1 / torch.sqrt(((r - r.mean(1, keepdim=True)) ** 2).mean(1, keepdim=True) + eps)
    ww = 1 if w is None else w.double().abs()
    bigh = bigh + big * f * ww
    return (r, big), (h, bigh)


def check(got, want, big, name):
    tol = U[got.dtype] * want.abs() + 2.0 ** -17 * big.amax(1, keepdim=True) + 2.0 ** -25
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} values off, worst {float((err / tol).max()):.2f} of the tolerance"


def strided(t, pad):
    if not pad:
        return t
    buf = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def case(t, d, dtype, rdtype, pdtype, kind, post, gates, pad, seed, weights=True, residual=True, mean=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s, dtype=dtype, mul=1.0, add=0.0):
        return (torch.randn(s, generator=g, device="cuda") * mul + add).to(dtype)

    x = strided(rnd(t, d, add=mean), pad)
    res = strided(rnd(t, d, dtype=rdtype, mul=2.0), pad) if residual else None
    gate = None if not gates else rnd(d, dtype=pdtype) if gates == 1 else rnd(gates, d, dtype=pdtype)
    pw, pb, w, b = ((rnd(d, dtype=pdtype, add=1.0) if weights else None) for _ in range(4))
    out = torch.full((t + 1, d), GUARD, dtype=dtype, device="cuda")
    r_out = torch.full((t + 1, d), GUARD, dtype=rdtype, device="cuda")
    r, h = qnn.block_norm(x, res, pre_weight=w, pre_bias=b, post_norm=post, post_weight=pw if post else None,
                          post_bias=pb if post else None, gate=gate, scale=0.7, eps=1e-5, kind=kind,
                          residual_out=r_out[:t], out=out[:t])
    (wr, br), (wh, bh) = reference(x, res, gate, post, pw, pb, w, b, 0.7, 1e-5, kind)
    if t:
        check(r, wr, br, "r")
        check(h, wh, bh, "h")
    assert bool((out[t:] == GUARD).all()) and bool((r_out[t:] == GUARD).all()), "wrote past the last row"


@pytest.mark.parametrize("t,d", [(0, 64), (1, 1), (1, 8), (3, 7), (2, 33), (5, 64), (4, 1000), (700, 257), (3, 2049),
                                 (9, 4096), (400, 4096), (350, 8192), (2, 16392), (3, 32768), (2, 32761)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_sizes(t, d, dtype, kind):
    case(t, d, dtype, dtype, dtype, kind, True, 1, 0, seed=t * 31 + d)


@pytest.mark.parametrize("pad", [0, 1, 8, 15])
@pytest.mark.parametrize("gates", [0, 1, 3])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("wide", ["same", "residual", "params", "both"])
def test_forms(pad, gates, post, wide):
    f32 = torch.float32
    case(12, 1032, torch.bfloat16, f32 if wide in ("residual", "both") else torch.bfloat16,
         f32 if wide in ("params", "both") else torch.bfloat16, "layer" if gates == 1 else "rms", post, gates, pad, seed=5)


@pytest.mark.parametrize("t,d", [(7304, 520), (4692, 1736), (1920, 4096), (930, 8192), (459, 16384)])
@pytest.mark.parametrize("gates", [0, 1, 3])
@pytest.mark.parametrize("kind,post,residual,weights", [("rms", False, True, True), ("rms", True, True, True),
                                                        ("layer", True, True, True), ("rms", False, False, False),
                                                        ("layer", False, True, False)])
@pytest.mark.parametrize("dtype,rdtype,pdtype", [(torch.bfloat16, torch.float32, torch.bfloat16),
                                                 (torch.float16, torch.float16, torch.float16),
                                                 (torch.bfloat16, torch.bfloat16, torch.float32),
                                                 (torch.float32, torch.float32, torch.float32)])
def test_many_rows(t, d, gates, kind, post, residual, weights, dtype, rdtype, pdtype):
    """Enough whole rows for the blocks that stay resident, in every combination of optional operands."""
    t = t // 3 * 3 if gates == 3 else t
    case(t, d, dtype, rdtype, pdtype, kind, post, gates, 0, seed=t + d, weights=weights, residual=residual)


def test_many_rows_strided_in_place_and_residual_only():
    base = torch.randn(4700, 1744, device="cuda").bfloat16()
    x, res = base[:, :1736], torch.randn(4700, 1736, device="cuda")
    r, h = qnn.block_norm(x, res, scale=0.5)
    r1, none = qnn.block_norm(x, res, scale=0.5, pre_norm=False)
    assert none is None and torch.equal(r1, r)
    x2, res2 = base.clone()[:, :1736], res.clone()
    qnn.block_norm(x2, res2, scale=0.5, residual_out=res2, out=x2)
    assert torch.equal(res2, r) and torch.equal(x2, h)


def test_no_weights_no_residual():
    case(6, 520, torch.float16, torch.float16, torch.float16, "rms", True, 0, 0, seed=1, weights=False, residual=False)
    case(6, 520, torch.bfloat16, torch.float32, torch.bfloat16, "layer", False, 0, 0, seed=2, weights=False, residual=False)


def test_large_mean_does_not_cancel():
    """A layer norm of rows whose mean is 1000 times their spread."""
    case(5, 4096, torch.float32, torch.float32, torch.float32, "layer", True, 0, 0, seed=3, mean=1000.0)


def test_in_place_and_residual_only():
    x = torch.randn(37, 1000, device="cuda").bfloat16()
    res = torch.randn(37, 1000, device="cuda")
    w = torch.randn(1000, device="cuda").bfloat16()
    r, h = qnn.block_norm(x, res, pre_weight=w, post_norm=True, scale=0.5)
    r1, none = qnn.block_norm(x, res, post_norm=True, scale=0.5, pre_norm=False)
    assert none is None and torch.equal(r1, r)
    x2, res2 = x.clone(), res.clone()
    r2, h2 = qnn.block_norm(x2, res2, pre_weight=w, post_norm=True, scale=0.5, residual_out=res2, out=x2)
    assert r2 is res2 and h2 is x2 and torch.equal(r2, r) and torch.equal(h2, h)


def test_nonfinite_rows_stay_alone():
    x = torch.randn(9, 777, device="cuda")
    res = torch.randn(9, 777, device="cuda")
    r, h = qnn.block_norm(x, res, post_norm=True)
    x2 = x.clone()
    x2[2, 5], x2[6, 700] = math.nan, math.inf
    r2, h2 = qnn.block_norm(x2, res, post_norm=True)
    rest = [i for i in range(9) if i not in (2, 6)]
    assert torch.equal(r2[rest], r[rest]) and torch.equal(h2[rest], h[rest])
    assert bool(h2[2].isnan().all()) and bool(h2[6].isnan().any())


def test_zero_rows_give_the_bias():
    x = torch.zeros(2, 100, device="cuda", dtype=torch.float16)
    b = torch.randn(100, device="cuda").half()
    for kind in ("rms", "layer"):
        r, h = qnn.block_norm(x, post_norm=True, pre_bias=b, kind=kind)
        assert bool((r == 0).all()) and torch.equal(h, b.expand(2, -1))


def test_another_stream():
    x = torch.randn(64, 512, device="cuda").bfloat16()
    want = qnn.block_norm(x, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = qnn.block_norm(x, x)
    got2 = qnn.block_norm(x, x, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, got2))


@pytest.mark.parametrize("kw,error", [
    (dict(gate=(5, 64)), ValueError), (dict(gate=(0, 64)), ValueError), (dict(residual=(4, 65)), ValueError),
    (dict(pre_weight=(63,)), ValueError), (dict(kind="batch"), ValueError), (dict(pre_weight=(64, torch.float64)), TypeError),
    (dict(pre_weight=(64, torch.float32), pre_bias=(64, torch.bfloat16)), TypeError), (dict(eps=-1.0), qnn.QnnError),
    (dict(residual_out=(4, 64, torch.float16)), TypeError), (dict(cols=2), ValueError), (dict(eps=math.nan), qnn.QnnError)])
def test_refusals(kw, error):
    kw = dict(kw)
    x = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)
    if "cols" in kw:
        x = torch.zeros(4, 64 * kw.pop("cols"), device="cuda", dtype=torch.bfloat16)[:, ::2]

    def make(v):
        if not isinstance(v, tuple):
            return v
        dt = v[-1] if isinstance(v[-1], torch.dtype) else torch.bfloat16
        return torch.zeros([n for n in v if not isinstance(n, torch.dtype)], device="cuda", dtype=dt)

    with pytest.raises(error):
        qnn.block_norm(x, **{k: make(v) for k, v in kw.items()})


def test_host_tensors_are_refused():
    with pytest.raises(ValueError):
        qnn.block_norm(torch.zeros(4, 64))
    with pytest.raises(qnn.QnnError) as e:
        qnn.block_norm(torch.zeros(1, 32769, device="cuda"))
    assert e.value.status == qnn.QNN_EUNSUPPORTED
