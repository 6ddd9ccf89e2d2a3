"""The products at sizes past those of test_gpu_matmul.py: long rows, single channels, and many experts.  Tolerances:
block_util.py."""
import pytest
import torch

from block_util import check, gen, product64, weights
from paper_1908_11263_gb300 import qnn
from test_gpu_matmul import BF, HF, routed, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,k,m", [(1, 33000, 40), (20, 20004, 33), (40, 33000, 1), (200, 16388, 260), (700, 8, 1)])
@pytest.mark.parametrize("bits", [16, 8, 4, 2])
def test_long_rows_and_single_channels(t, k, m, bits):
    run(t, k, m, bits, BF if bits in (16, 4) else HF, gated=bits == 8, act="silu" if bits == 8 else "none", bias=True, residual=True)


@pytest.mark.parametrize("t,top,experts", [(1, 8, 65), (40, 8, 200), (300, 4, 512), (2500, 8, 1024), (4000, 1, 129)])
@pytest.mark.parametrize("bits", [16, 4])
def test_many_experts(t, top, experts, bits):
    k, m, g = 136, 72, gen(t + experts + bits)
    w, scale, w64 = weights(m, k, bits, BF, g, experts)
    layer = qnn.PreparedExperts(w, scale=scale, bits=bits, dtype=BF, act="relu")
    ids, cw = routed(t, top, experts, g, dropped=0.1)
    plan = qnn.expert_plan(ids, experts)
    off, order = plan.offsets.tolist(), plan.order.long()
    x = torch.randn(t, k, generator=g, device="cuda").to(BF)
    y = layer.dispatch(x, plan)
    h = torch.randn(t * top, k, generator=g, device="cuda").to(BF)
    z = layer.combine(h, plan, cw)
    want = torch.zeros(t, m, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(want)
    for e in range(experts):
        if off[e] == off[e + 1]:
            continue
        slots, places = order[off[e]:off[e + 1]], slice(off[e], off[e + 1])
        s = None if scale is None else scale[e]
        check(y[places], *product64(x[slots // top], w64[e], s, None, m, False, "relu"), f"expert {e}")
        v, ev = product64(h[places], w64[e], s, None, m, False, "relu")
        f = cw.reshape(-1)[slots].double()[:, None]
        want.index_add_(0, slots // top, f * v)
        err.index_add_(0, slots // top, f * (ev + (top + 1) * 2.0 ** -24 * v.abs()))
    check(z, want, err, "combine")
    assert bool((y[off[-1]:] == 0).all())
