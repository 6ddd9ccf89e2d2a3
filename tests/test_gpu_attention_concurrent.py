"""Attention calls of every kernel on several streams at once, beside products that hold tensor memory too."""
import pytest
import torch

from attention_util import gen, randn
from paper_1908_11263_gb300 import qnn
from test_gpu_attention import paged

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def calls():
    g = gen(77)
    few = paged(g, BF, [1] * 30, [600 + 40 * i for i in range(30)], 8, 2, 128, 16)
    short = paged(g, F16, [400, 30, 1, 700], [900, 30, 500, 2000], 4, 2, 64, 24)
    long = paged(g, BF, [1500, 20], [4000, 900], 8, 2, 128, 32)
    wide = paged(g, BF, [90, 40], [300, 900], 4, 2, 256, 16)
    both = paged(g, BF, [1, 1, 200] * 4, [700, 90, 400] * 4, 2, 2, 64, 16)  # each kernel its own sequences
    both = both[0], both[1][:8].contiguous(), both[2][:8].contiguous(), torch.tensor([0, 1, 2, 60, 61, 62, 63, 64, 65], dtype=torch.int32,
                                                                                     device="cuda"), both[4][:66]
    qc, kc, vc = randn(g, 4, 300, 8, 64), randn(g, 4, 700, 8, 64), randn(g, 4, 700, 8, 64)
    product, x = qnn.PreparedMatmul(randn(g, 2048, 1024, mul=0.03)), randn(g, 1000, 1024)
    each = [lambda s, c=c: c[0].attend(c[4], c[1], c[2], c[3], lse=True, stream=s) for c in (few, short, long, wide)]
    each.append(lambda s: both[0].attend(both[4], both[1], both[2], both[3], lse=True, stream=s))
    each.append(lambda s: qnn.cross_attention(qc, kc, vc, lse=True, stream=s))
    each.append(lambda s: (product(x, stream=s),))
    return each


def test_streams_at_once():
    each = calls()
    want = [[o.clone() for o in f(None)] for f in each]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = []
    for i in range(12):
        for j, s in enumerate(streams):
            k = (i + 2 * j) % len(each)
            got.append((k, each[k](s)))
    torch.cuda.synchronize()
    qnn.device_status()
    for k, outs in got:
        # rows in no sequence are not written: the last of the fifth call's 66
        assert all(torch.equal(a[:65] if k == 4 else a, b[:65] if k == 4 else b) for a, b in zip(outs, want[k])), k
