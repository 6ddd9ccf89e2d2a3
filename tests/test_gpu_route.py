"""qnn.route_topk and qnn.expert_plan against plain implementations in 64 bits and whole numbers.

Tolerances: a score passes one exponential (2 ulp), a division and, for softmax, a sum of at most 1024 terms in a tree
(37 roundings a term): under 64 roundings of 2^-24, 4e-6; renormalising adds the same again.  Two candidates closer than
that may change places; where scores are equal by construction the order has to be exact."""
import math

import numpy as np
import pytest
import torch

from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
TOL = 8e-6


def reference_row(x, k, score, bias, groups, top_groups, group_score, renorm, scale):
    """One token: (weights, ids, what the choice went by) from the definitions."""
    open_ = [i for i, v in enumerate(x) if v > -math.inf]  # NaN compares false
    s = [0.0] * len(x)
    if score == "sigmoid":
        for i in open_:
            s[i] = 0.0 if x[i] < -700 else 1 / (1 + math.exp(-x[i]))
    elif open_:
        top = max(x[i] for i in open_)
        ex = {i: math.exp(x[i] - top) if top < math.inf else float(x[i] == math.inf) for i in open_}
        for i in open_:
            s[i] = ex[i] / sum(ex.values())
    pick = {i: s[i] + (0.0 if bias is None else bias[i]) for i in open_}
    if score == "softmax" and bias is None:
        order = {i: x[i] for i in open_}  # the same order, without rounding
    else:
        order = dict(pick)
    size = len(x) // groups
    if top_groups < groups:
        of = []
        for g in range(groups):
            v = sorted((pick[i] for i in range(g * size, (g + 1) * size) if i in pick), reverse=True)
            of.append(-math.inf if not v else sum(v[:2]) if group_score == "top2" else v[0])
        keep = sorted(range(groups), key=lambda g: (-of[g], g))[:top_groups]
        order = {i: v for i, v in order.items() if i // size in keep}
    ids = sorted(order, key=lambda i: (-order[i], i))[:k]
    w = [s[i] for i in ids]
    if renorm and sum(w) > 0:
        w = [v / sum(w) for v in w]
    w = [v * scale for v in w]
    pad = k - len(ids)
    return w + [0.0] * pad, ids + [-1] * pad, pick


def check(x, k, exact_order=False, **kw):
    full = dict(score="softmax", bias=None, groups=1, top_groups=None, group_score="max", renormalise=True, scale=1.0)
    full.update(kw)
    w, ids = qnn.route_topk(x, k, **full)
    assert w.shape == ids.shape == (x.shape[0], k) and w.dtype == torch.float32 and ids.dtype == torch.int32
    xs, ws, got = x.double().cpu().numpy(), w.double().cpu().numpy(), ids.cpu().numpy()
    bias = None if full["bias"] is None else full["bias"].double().cpu().numpy()
    for t in range(x.shape[0]):
        rw, rid, pick = reference_row(xs[t], k, full["score"], bias, full["groups"], full["top_groups"] or full["groups"],
                                      full["group_score"], full["renormalise"], full["scale"])
        if exact_order or list(got[t]) == rid:
            assert list(got[t]) == rid, (t, got[t], rid)
        else:  # the same scores in the same order up to rounding, no expert twice
            assert len(set(got[t])) == k and (got[t] >= 0).sum() == (np.array(rid) >= 0).sum()
            assert all(abs(pick[a] - pick[b]) <= TOL * max(1, abs(pick[b])) for a, b in zip(got[t], rid)), (t, got[t], rid)
        assert np.allclose(ws[t], rw, rtol=TOL, atol=TOL * abs(full["scale"])), (t, ws[t], rw)


def logits(t, e, seed, dtype=torch.float32, closed=0.0, empty=()):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, e, generator=g, device="cuda") * 2
    if closed:
        x[torch.rand(t, e, generator=g, device="cuda") < closed] = -math.inf
    for i in empty:
        x[i] = -math.inf
    return x.to(dtype)


@pytest.mark.parametrize("t,e,k", [(0, 8, 2), (1, 1, 1), (1, 8, 8), (3, 33, 5), (9, 64, 4), (17, 100, 32), (65, 256, 8),
                                   (5, 1000, 16), (4, 1024, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_sizes(t, e, k, score, dtype):
    check(logits(t, e, t + e, dtype), k, score=score, renormalise=bool(e % 2), scale=2.5)


@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 2), (8, 1), (8, 7), (32, 3)])
@pytest.mark.parametrize("group_score", ["max", "top2"])
@pytest.mark.parametrize("score,biased", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
def test_groups_and_bias(groups, top_groups, group_score, score, biased):
    x = logits(33, 96, groups * 7 + top_groups, closed=0.3, empty=(0, 32))
    bias = torch.linspace(-0.5, 0.5, 96, device="cuda").roll(17) if biased else None
    check(x, 3, score=score, bias=bias, groups=groups, top_groups=top_groups, group_score=group_score)


def test_ties_go_to_the_lowest_index():
    x = torch.randint(-2, 3, (50, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
    check(x, 8, exact_order=True)
    check(x, 8, exact_order=True, groups=8, top_groups=3)
    check(torch.zeros(3, 40, device="cuda"), 32, exact_order=True, score="sigmoid", groups=4, top_groups=4)
    z = torch.zeros(2, 6, device="cuda")
    z[:, ::2] = -0.0  # the zeros are equal
    check(z, 4, exact_order=True)


def test_closed_experts_and_empty_rows():
    x = logits(40, 16, 3, closed=0.85, empty=(0, 7, 39))
    x[5, 3] = math.nan
    x[6] = math.nan
    for score in ("softmax", "sigmoid"):
        check(x, 6, score=score)
    w, ids = qnn.route_topk(x, 6)
    for t in (0, 6, 7, 39):
        assert bool((ids[t] == -1).all()) and bool((w[t] == 0).all())


def test_extreme_logits():
    low = torch.finfo(torch.float32).min
    x = logits(6, 12, 8)
    x[0] = low                      # lowest finite values are open and equal
    x[1, 4] = math.inf
    x[2, 3], x[2, 9] = math.inf, math.inf
    x[3] = torch.linspace(-300, 300, 12)
    x[4, 2] = low
    check(x[:3], 4, exact_order=True)
    check(x, 4)
    check(x[3:], 4, score="sigmoid")


def test_strided_logits():
    base = logits(20, 80, 4)
    base[:, 64:] = math.nan
    a = qnn.route_topk(base[:, :64], 5)
    b = qnn.route_topk(base[:, :64].contiguous(), 5)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("tokens,top,experts", [(0, 4, 8), (1, 1, 1), (31, 1, 7), (512, 4, 64), (1025, 2, 257), (3, 5, 1024),
                                                (40000, 8, 128), (300001, 1, 1000)])
def test_plan(tokens, top, experts):
    rng = np.random.default_rng(tokens + experts)
    ids = rng.integers(-1, experts + 1, size=(tokens, top)).astype(np.int32)  # -1 and `experts` go nowhere
    if tokens > 100:
        ids[: tokens // 3] = experts // 2  # one crowded expert
    plan = qnn.expert_plan(torch.from_numpy(ids).cuda(), experts)
    flat = ids.reshape(-1)
    live = (flat >= 0) & (flat < experts)
    order = np.argsort(np.where(live, flat, experts), kind="stable")[: live.sum()]
    want = np.full(flat.size, -1)
    want[: order.size] = order
    position = np.full(flat.size, -1)
    position[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[live], minlength=experts))])
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    assert np.array_equal(plan.order.cpu().numpy(), want)
    assert np.array_equal(plan.position.cpu().numpy().reshape(-1), position)
    assert (plan.tokens, plan.top, plan.experts) == (tokens, top, experts)


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    for kw in (dict(k=0), dict(k=65), dict(k=2, groups=5), dict(k=2, groups=4, top_groups=5), dict(k=2, scale=math.inf)):
        with pytest.raises(qnn.QnnError) as e:
            qnn.route_topk(x, **kw)
        assert e.value.status == qnn.QNN_EINVAL
    for bad, k in ((torch.zeros(1, 1025, device="cuda"), 2), (x, 33)):
        with pytest.raises(qnn.QnnError) as e:
            qnn.route_topk(bad, k)
        assert e.value.status == qnn.QNN_EUNSUPPORTED
    with pytest.raises(ValueError):
        qnn.route_topk(x, 2, score="tanh")
    with pytest.raises(ValueError):
        qnn.route_topk(x, 2, bias=torch.zeros(63, device="cuda"))
    with pytest.raises(TypeError):
        qnn.route_topk(x, 2, bias=torch.zeros(64, device="cuda", dtype=torch.float16))
    with pytest.raises(TypeError):
        qnn.route_topk(x.long(), 2)
    with pytest.raises(TypeError):
        qnn.expert_plan(torch.zeros(4, 2, device="cuda", dtype=torch.int64), 8)
    with pytest.raises(ValueError):
        qnn.expert_plan(torch.zeros(4, device="cuda", dtype=torch.int32), 8)
    for experts, status in ((0, qnn.QNN_EINVAL), (1025, qnn.QNN_EUNSUPPORTED)):
        with pytest.raises(qnn.QnnError) as e:
            qnn.expert_plan(torch.zeros(4, 2, device="cuda", dtype=torch.int32), experts)
        assert e.value.status == status
