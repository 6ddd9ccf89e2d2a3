"""Sizes past what the product kernels' 32-bit counters hold are refused with QNN_EUNSUPPORTED, by the size queries too and
before anything is queued; the largest sizes that the header names are counted within 32 bits.  No GPU: refusals come before
any CUDA call."""
import ctypes

import pytest

from paper_1908_11263_gb300 import build as qbuild
from paper_1908_11263_gb300 import qnn
from test_block_boundary import FAKE, matmul_desc, size_of

HUGE = (1 << 64) - 1  # bytes of an image


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    return qnn.load()


@pytest.mark.parametrize("kw,status", [
    (dict(m=1 << 24, k=1 << 16, bits=2), qnn.QNN_OK), (dict(m=1 << 16, k=1 << 24, bits=2), qnn.QNN_OK),
    (dict(m=(1 << 24) - 31, k=1 << 16, bits=16), qnn.QNN_OK),
    (dict(m=1 << 24, k=(1 << 16) + 4, bits=2), qnn.QNN_EUNSUPPORTED),
    (dict(m=1 << 24, k=1 << 16, bits=4, gated=1), qnn.QNN_EUNSUPPORTED),
    (dict(experts=1024, m=1 << 20, k=1 << 10, bits=8), qnn.QNN_OK),
    (dict(experts=1024, m=1 << 20, k=(1 << 10) + 1, bits=8), qnn.QNN_EUNSUPPORTED),
    (dict(experts=1024, m=1 << 24, k=4, bits=2), qnn.QNN_OK),            # columns count in 64s
    (dict(experts=1024, m=1 << 24, k=4, bits=2, gated=1), qnn.QNN_EUNSUPPORTED)])
def test_weights(lib, kw, status):
    d = ctypes.byref(matmul_desc(**kw))
    assert size_of(lib.qnn_matmul_image_size, d)[0] == status
    if status != qnn.QNN_OK:
        assert lib.qnn_matmul_prepare(d, FAKE, None, None, FAKE, HUGE, None) == status
        assert lib.qnn_matmul_run(d, FAKE, HUGE, 1, FAKE, 1 << 24, None, 0, FAKE, 1 << 24, 0, None, 0, None) in (status, qnn.QNN_EINVAL)


@pytest.mark.parametrize("t,m,status", [(1 << 20, 1 << 18, qnn.QNN_OK), (1 << 20, (1 << 18) + 1, qnn.QNN_EUNSUPPORTED),
                                        (1 << 14, 1 << 24, qnn.QNN_OK), ((1 << 14) + 1, 1 << 24, qnn.QNN_EUNSUPPORTED)])
def test_outputs(lib, t, m, status):
    d = ctypes.byref(matmul_desc(m=m, k=64))
    assert size_of(lib.qnn_matmul_workspace_size, d, t, FAKE, 64)[0] == status
    if status != qnn.QNN_OK:
        assert lib.qnn_matmul_run(d, FAKE, HUGE, t, FAKE, 64, None, 0, FAKE, m, 0, FAKE, HUGE, None) == status
    e = ctypes.byref(matmul_desc(experts=2, m=m, k=64))
    for combine in (0, 1):
        assert size_of(lib.qnn_experts_workspace_size, e, t, 1, combine, FAKE, 64)[0] == status
    if status != qnn.QNN_OK:
        assert lib.qnn_experts_dispatch(e, FAKE, HUGE, t, 1, FAKE, FAKE, FAKE, 64, FAKE, m, FAKE, HUGE, None) == status
        assert lib.qnn_experts_combine(e, FAKE, HUGE, t, 1, FAKE, FAKE, FAKE, FAKE, 64, None, 0, FAKE, m, FAKE, HUGE, None) == status


def test_counters_hold_the_largest_sizes():
    """The kernels' counters at the limits: tiles of x times image tiles, and units times their blocks along K, stay below
    2^31 (2^30 where a counter is doubled), over the corners of what the checks let through."""
    sizes = [1, 2, 31, 1024, 1 << 14, 1 << 20, 1 << 24]
    for experts in (1, 2, 100, 1024):
        for m in sizes:
            for k in sizes:
                for gated in (0, 1):
                    rows = (m + 7) // 8 * 16 if gated else m
                    mb, kb, mt = -(-rows // 32), -(-k // 64), -(-rows // 256)
                    if experts * mb * kb > 1 << 29:
                        continue
                    for t in (1, 32, 33, 6 * experts, 16 * experts, 1 << 14, 1 << 20):
                        t = min(t, (1 << 38) // m, 1 << 20)
                        if t == 0:
                            continue
                        live = min(experts, t)
                        assert (-(-t // 16) + live) * mt < 1 << 30                # tensor cores, the narrowest tiles
                        if t <= (16 * experts if experts > 1 else 32):            # streamed
                            want = -(-t // experts)
                            nt = 8 if want <= 8 else 16 if want <= 16 else 32
                            assert (-(-t // nt) + live) * mb * -(-kb // 8) < 1 << 31
