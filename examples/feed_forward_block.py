"""One feed-forward block of a decoder with experts, as it is served: the block operators in the order a model calls them.

    residual stream r, output a of the attention before it
      r, h    = block_norm(a, r)                    norm after, gate, residual sum, norm before
      logits  = router(h)                           16-bit product with 32-bit outputs
      w, ids  = route_topk(logits)                  k experts a token, balance bias, limited groups
      plan    = expert_plan(ids)
      u       = up.dispatch(h, plan)                gated product, INT-4 weights
      y       = down.combine(u, plan, w, shared(h)) INT-8 weights, weighted sum, shared expert's output added
      r, h    = block_norm(y, r)                    into the next block

Run it:  python examples/feed_forward_block.py [tokens]   (default 16, a decode batch)
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1908_11263_gb300 import qnn  # noqa: E402


def packed(rows, k, bits, g, experts=None):
    """Random packed codes and scales that keep products near one."""
    shape = ((experts,) if experts else ()) + (rows, k)
    w = torch.randint(0, 256, shape[:-1] + (k * bits // 8,), generator=g, device="cuda", dtype=torch.uint8)
    rms = math.sqrt((4.0 ** bits + 2) / 12)
    return w, (0.5 + torch.rand(shape[:-1], generator=g, device="cuda")) / (rms * math.sqrt(k))


class FeedForwardBlock:
    """Weights of the block, laid out once."""

    def __init__(self, width=512, hidden=256, experts=16, top=4, groups=4, top_groups=2, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def rnd(*s, mul=1.0, add=0.0):
            return torch.randn(s, generator=g, device="cuda") * mul + add

        self.top, self.groups, self.top_groups, self.experts = top, groups, top_groups, experts
        self.post_weight, self.pre_weight = rnd(width, mul=0.1, add=1).bfloat16(), rnd(width, mul=0.1, add=1).bfloat16()
        self.gate = rnd(width).bfloat16()
        self.router_weight = rnd(experts, width, mul=1 / math.sqrt(width)).bfloat16()
        self.router_bias = rnd(experts, mul=0.1)
        self.up_codes, self.up_scale = packed(2 * hidden, width, 4, g, experts)
        self.down_codes, self.down_scale = packed(width, hidden, 8, g, experts)
        self.shared_up_weight = rnd(2 * hidden, width, mul=1 / math.sqrt(width)).bfloat16()
        self.shared_down_codes, self.shared_down_scale = packed(width, hidden, 8, g)
        self.router = qnn.PreparedMatmul(self.router_weight)
        self.up = qnn.PreparedExperts(self.up_codes, scale=self.up_scale, bits=4, gated=True, act="silu")
        self.down = qnn.PreparedExperts(self.down_codes, scale=self.down_scale, bits=8)
        self.shared_up = qnn.PreparedMatmul(self.shared_up_weight, gated=True, act="silu")
        self.shared_down = qnn.PreparedMatmul(self.shared_down_codes, scale=self.shared_down_scale, bits=8)

    def __call__(self, attention, residual):
        """attention [t, width] bfloat16, residual [t, width] float32; returns the new residual and the next block's input."""
        residual, h = qnn.block_norm(attention, residual, post_norm=True, post_weight=self.post_weight, gate=self.gate,
                                     pre_weight=self.pre_weight)
        logits = self.router(h, out_dtype=torch.float32)
        weights, ids = qnn.route_topk(logits, self.top, score="sigmoid", bias=self.router_bias, groups=self.groups,
                                      top_groups=self.top_groups, group_score="top2")
        plan = qnn.expert_plan(ids, self.experts)
        y = self.down.combine(self.up.dispatch(h, plan), plan, weights, residual=self.shared_down(self.shared_up(h)))
        return qnn.block_norm(y, residual, pre_weight=self.pre_weight)


def main():
    tokens = int(sys.argv[1]) if len(sys.argv) > 1 else 16
    block = FeedForwardBlock()
    a = torch.randn(tokens, 512, device="cuda").bfloat16()
    r = torch.randn(tokens, 512, device="cuda")
    new_r, h = block(a, r)
    qnn.device_status()
    print(f"{tokens} tokens: residual {tuple(new_r.shape)} {new_r.dtype}, next input {tuple(h.shape)} {h.dtype}, "
          f"rms {float(h.float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
