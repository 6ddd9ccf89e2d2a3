"""qnn.expert_plan for every number of experts around the default limit of a block's shared memory (48 KB, static memory
included; the placing kernel takes 72 bytes an expert).  In a process of its own: a call with more experts raises the limit
for the calls after it, so the numbers go up."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import numpy as np
import torch
from paper_1908_11263_gb300 import qnn
for tokens in (50, 3000):
    for experts in (679, 680, 681, 682, 683, 684):
        ids = np.random.default_rng(experts).integers(-1, experts + 1, size=(tokens, 2)).astype(np.int32)
        plan = qnn.expert_plan(torch.from_numpy(ids).cuda(), experts)
        flat = ids.reshape(-1)
        live = (flat >= 0) & (flat < experts)
        order = np.argsort(np.where(live, flat, experts), kind="stable")[: live.sum()]
        got = plan.order.cpu().numpy()
        assert np.array_equal(got[: order.size], order) and (got[order.size:] == -1).all(), experts
        offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[live], minlength=experts))])
        assert np.array_equal(plan.offsets.cpu().numpy(), offsets), experts
        print("ok", tokens, experts, flush=True)
"""


def test_numbers_of_experts_around_the_shared_memory_limit():
    r = subprocess.run([sys.executable, "-c", PROGRAM], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-500:] + r.stderr[-2000:]
    assert r.stdout.count("ok") == 12
