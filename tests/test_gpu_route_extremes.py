"""qnn.route_topk where scores underflow in 32 bits: logits far below the row's largest, and scores that are all tiny.  The
reference is the definition in 64 bits (exp(-250) is 2.7e-109 there); its weights and tolerance are those of
test_gpu_route.py.  The values are spread so that no two groups or experts that compete are within 1e-3 of one another."""
import math

import numpy as np
import pytest
import torch

from paper_1908_11263_gb300 import qnn
from test_gpu_route import TOL, logits, reference_row

pytestmark = pytest.mark.gpu


def check(x, k, **kw):
    full = dict(score="softmax", bias=None, groups=1, top_groups=None, group_score="max", renormalise=True, scale=1.0)
    full.update(kw)
    w, ids = qnn.route_topk(x, k, **full)
    bias = None if full["bias"] is None else full["bias"].double().cpu().numpy()
    xs = x.double().cpu().numpy()
    for t in range(x.shape[0]):
        rw, rid, _ = reference_row(xs[t], k, full["score"], bias, full["groups"], full["top_groups"] or full["groups"],
                                   full["group_score"], full["renormalise"], full["scale"])
        assert ids[t].tolist() == rid, (t, ids[t], rid)
        assert np.allclose(w[t].double().cpu().numpy(), rw, rtol=TOL, atol=TOL * abs(full["scale"])), (t, w[t], rw)


def far_groups(t, groups, size, near, seed):
    """Groups in random order: `near` of them around zero, the others 150 to 250 below, one step of 10 apart."""
    x = logits(t, groups * size, seed).clamp(-4, 4).view(t, groups, size) * 0.1
    rng = np.random.default_rng(seed)
    for i in range(t):
        for n, g in enumerate(rng.permutation(groups)):
            x[i, g] += 3.0 * n if n < near else -150.0 - 10.0 * n
    return x.view(t, groups * size)


@pytest.mark.parametrize("groups,size,top_groups", [(8, 8, 4), (8, 12, 5), (4, 24, 3), (16, 2, 9), (32, 1, 6)])
@pytest.mark.parametrize("shift", [0.0, 500.0, -1e6])  # softmax does not change with it
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_groups_far_below_the_best(groups, size, top_groups, shift, group_score):
    x = far_groups(33, groups, size, 1, groups + size)
    if shift == -1e6:
        x = (x * 16).round() / 16  # exact after the shift
    check(x + shift, min(32, size * top_groups), groups=groups, top_groups=top_groups, group_score=group_score)


def test_far_groups_keep_their_two_best():
    """Of far groups the sum of two counts, not the best alone: two at -200 are more than one at -199.5 with nothing beside."""
    x = torch.full((2, 12), -math.inf, device="cuda")
    x[:, 0] = 0.0
    x[:, 3] = -199.5
    x[:, 6:8] = -200.0
    x[1, 9:11] = -199.9
    check(x, 4, groups=4, top_groups=2, group_score="top2")
    _, ids = qnn.route_topk(x, 3, groups=4, top_groups=2, group_score="top2")
    assert ids.tolist() == [[0, 6, 7], [0, 9, 10]]


def test_closed_groups_stay_closed():
    x = torch.full((1, 8), -math.inf, device="cuda")
    x[0, 1], x[0, 6] = 0.0, -3e38
    w, ids = qnn.route_topk(x, 3, groups=4, top_groups=3, group_score="top2")
    assert ids.tolist() == [[1, 6, -1]] and w.tolist() == [[1.0, 0.0, 0.0]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_shares_of_chosen_experts_that_all_underflow(score):
    """A balance bias may choose experts whose scores are all tiny; their shares add up to one all the same."""
    x = logits(40, 64, 5).clamp(-4, 4)
    bias = torch.zeros(64, device="cuda")
    far = torch.arange(3, 64, 9, device="cuda")
    if score == "softmax":
        x[:, far] -= 180.0
    else:
        x -= 180.0
    bias[far] = 10.0 + torch.arange(far.numel(), device="cuda")
    check(x, 5, score=score, bias=bias, scale=2.5)


def test_an_infinite_logit_leaves_the_others_nothing():
    x = logits(3, 16, 6)
    x[:, 2] = math.inf
    bias = torch.zeros(16, device="cuda")
    bias[8:] = 10.0
    w, ids = qnn.route_topk(x, 4, bias=bias)
    assert bool((ids >= 8).all()) and bool((w == 0).all())
