"""The example's feed-forward block against the same block written with plain 64-bit products.

Tolerance: every step of the library rounds its output to bfloat16 (2^-8 of it at most, 2^-9.8 in the root mean square); the
next block's input lies behind six such roundings (h, u, the shared expert's two, y, the output), each carried on by
products that keep relative errors of independent terms as they are: 6 * 2^-9.8 < 0.007 of the root mean square; three times
that is allowed.  The experts are chosen from the library's own 32-bit logits on both sides, so no near tie can differ."""
import importlib.util
import os

import pytest
import torch

from block_util import act64
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("feed_forward_block", os.path.join(ROOT, "examples", "feed_forward_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def unpack(w, scale, bits):
    v = qnn.unpack_subbyte(w, bits, True) if bits < 8 else w.view(torch.int8)
    return v.double() * scale.double()[..., None]


def norm(v, w):
    return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w.double()


@pytest.mark.parametrize("tokens", [1, 16, 300, 1500])
def test_block(tokens):
    block = load_example().FeedForwardBlock()
    g = torch.Generator(device="cuda").manual_seed(tokens)
    a = torch.randn(tokens, 512, device="cuda", generator=g).bfloat16()
    r = torch.randn(tokens, 512, device="cuda", generator=g)
    got_r, got_h = block(a, r)
    qnn.device_status()

    _, h16 = qnn.block_norm(a, r, post_norm=True, post_weight=block.post_weight, gate=block.gate, pre_weight=block.pre_weight)
    weights, ids = qnn.route_topk(block.router(h16, out_dtype=torch.float32), block.top, score="sigmoid", bias=block.router_bias,
                                  groups=block.groups, top_groups=block.top_groups, group_score="top2")
    r64 = r.double() + block.gate.double() * norm(a.double(), block.post_weight)
    h = norm(r64, block.pre_weight)
    up, down = unpack(block.up_codes, block.up_scale, 4), unpack(block.down_codes, block.down_scale, 8)
    hidden = up.shape[1] // 2
    v = torch.einsum("tk,emk->tem", h, up)
    u = act64(v[..., :hidden], "silu") * v[..., hidden:]
    z = torch.einsum("tek,emk->tem", u, down)
    y = (z.gather(1, ids.long()[..., None].expand(-1, -1, z.shape[2])) * weights.double()[..., None]).sum(1)
    s = h @ block.shared_up_weight.double().t()
    y = y + (act64(s[:, :hidden], "silu") * s[:, hidden:]) @ unpack(block.shared_down_codes, block.shared_down_scale, 8).t()
    r64 = r64 + y
    h = norm(r64, block.pre_weight)
    for got, want in ((got_r, r64), (got_h, h)):
        err = float((got.double() - want).square().mean().sqrt() / want.square().mean().sqrt())
        assert err < 0.021, err
