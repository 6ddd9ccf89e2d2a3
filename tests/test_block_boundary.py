"""C ABI of the language-model block operators without a GPU: struct layouts, sizes, and the refusals that come before any
CUDA call (the pointers are never read)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_1908_11263_gb300 import build as qbuild
from paper_1908_11263_gb300 import qnn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # 256-byte aligned, never read


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    return qnn.load()


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "sizes.c"
    lines = []
    for struct, cls in (("qnn_norm_desc", qnn.NormDesc), ("qnn_route_desc", qnn.RouteDesc), ("qnn_matmul_desc", qnn.MatmulDesc)):
        lines.append(f'printf("%zu ", sizeof({struct}));')
        lines += [f'printf("%zu ", offsetof({struct}, {f}));' for f, _ in cls._fields_]
    src.write_text('#include <stdio.h>\n#include "qnn.h"\nint main(void) {' + "\n".join(lines) + "return 0;}\n")
    exe = tmp_path / "sizes"
    subprocess.run([cc, "-std=c99", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in (qnn.NormDesc, qnn.RouteDesc, qnn.MatmulDesc):
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def norm_desc(**kw):
    d = dict(kind=0, dtype=qnn.BF16, residual_dtype=qnn.BF16, param_dtype=qnn.BF16, post_norm=0, gates=1, d=64, t=4, ldx=64,
             ldres=64, ldr=64, ldh=64, scale=1.0, eps=1e-6)
    size = kw.pop("struct_size", ctypes.sizeof(qnn.NormDesc))
    d.update(kw)
    return qnn.NormDesc(size, *(d[f] for f, _ in qnn.NormDesc._fields_[1:]))


@pytest.mark.parametrize("kw,args,status", [
    (dict(struct_size=4), {}, qnn.QNN_EINVAL), (dict(kind=2), {}, qnn.QNN_EINVAL), (dict(dtype=3), {}, qnn.QNN_EINVAL),
    (dict(d=0), {}, qnn.QNN_EINVAL), (dict(t=-1), {}, qnn.QNN_EINVAL), (dict(ldx=63), {}, qnn.QNN_EINVAL),
    (dict(ldh=63), {}, qnn.QNN_EINVAL), (dict(ldres=63), dict(res=FAKE), qnn.QNN_EINVAL),
    (dict(gates=3), dict(gate=FAKE), qnn.QNN_EINVAL), (dict(gates=0), dict(gate=FAKE), qnn.QNN_EINVAL),
    (dict(eps=-1.0), {}, qnn.QNN_EINVAL), (dict(eps=float("inf")), {}, qnn.QNN_EINVAL), (dict(post_norm=2), {}, qnn.QNN_EINVAL),
    ({}, dict(x=None), qnn.QNN_EINVAL), ({}, dict(r=None, h=None), qnn.QNN_EINVAL),
    (dict(residual_dtype=qnn.F16), {}, qnn.QNN_EUNSUPPORTED), (dict(param_dtype=qnn.F16), {}, qnn.QNN_EUNSUPPORTED),
    (dict(d=32769, ldx=32769, ldr=32769, ldh=32769), {}, qnn.QNN_EUNSUPPORTED),
    ({}, dict(x=FAKE + 1), qnn.QNN_EALIGN), (dict(residual_dtype=qnn.F32), dict(r=FAKE + 2), qnn.QNN_EALIGN),
    ({}, dict(gate=FAKE + 1), qnn.QNN_EALIGN)])
def test_norm_refusals(lib, kw, args, status):
    a = dict(x=FAKE, res=None, gate=None, r=FAKE, h=FAKE)
    a.update(args)
    assert lib.qnn_block_norm(ctypes.byref(norm_desc(**kw)), a["x"], a["res"], a["gate"], None, None, None, None, a["r"], a["h"],
                              None) == status


def route_desc(**kw):
    d = dict(dtype=qnn.F32, experts=64, k=4, score=0, groups=1, top_groups=1, group_score=0, renormalise=1, scale=1.0, t=4, ld=64)
    d.update(kw)
    return qnn.RouteDesc(ctypes.sizeof(qnn.RouteDesc), *(d[f] for f, _ in qnn.RouteDesc._fields_[1:]))


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), qnn.QNN_EINVAL), (dict(k=65), qnn.QNN_EINVAL), (dict(experts=0), qnn.QNN_EINVAL), (dict(ld=63), qnn.QNN_EINVAL),
    (dict(groups=7), qnn.QNN_EINVAL), (dict(groups=4, top_groups=0), qnn.QNN_EINVAL), (dict(groups=4, top_groups=5), qnn.QNN_EINVAL),
    (dict(score=2), qnn.QNN_EINVAL), (dict(group_score=2), qnn.QNN_EINVAL), (dict(scale=float("nan")), qnn.QNN_EINVAL),
    (dict(t=-1), qnn.QNN_EINVAL), (dict(dtype=9), qnn.QNN_EINVAL), (dict(k=33), qnn.QNN_EUNSUPPORTED),
    (dict(experts=1025, ld=1025), qnn.QNN_EUNSUPPORTED), (dict(groups=64), qnn.QNN_EUNSUPPORTED)])
def test_route_refusals(lib, kw, status):
    assert lib.qnn_route_topk(ctypes.byref(route_desc(**kw)), FAKE, None, FAKE, FAKE, None) == status


def test_route_pointers(lib):
    d = ctypes.byref(route_desc())
    assert lib.qnn_route_topk(None, FAKE, None, FAKE, FAKE, None) == qnn.QNN_EINVAL
    assert lib.qnn_route_topk(d, None, None, FAKE, FAKE, None) == qnn.QNN_EINVAL
    assert lib.qnn_route_topk(d, FAKE + 2, None, FAKE, FAKE, None) == qnn.QNN_EALIGN
    assert lib.qnn_route_topk(d, FAKE, FAKE + 1, FAKE, FAKE, None) == qnn.QNN_EALIGN


def size_of(call, *args):
    n = ctypes.c_size_t(0)
    return call(*args, ctypes.byref(n)), n.value


def test_plan_sizes_and_refusals(lib):
    assert size_of(lib.qnn_expert_plan_workspace_size, 2048, 64) == (qnn.QNN_OK, 0)
    st, need = size_of(lib.qnn_expert_plan_workspace_size, 1 << 20, 64)
    assert st == qnn.QNN_OK and 0 < need <= 128 * 64 * 4
    assert size_of(lib.qnn_expert_plan_workspace_size, -1, 64)[0] == qnn.QNN_EINVAL
    assert size_of(lib.qnn_expert_plan_workspace_size, 8, 1025)[0] == qnn.QNN_EUNSUPPORTED
    assert size_of(lib.qnn_expert_plan_workspace_size, 1 << 31, 8)[0] == qnn.QNN_EUNSUPPORTED
    plan = lambda ids, slots, off, order, pos, ws, n: lib.qnn_expert_plan(ids, slots, 64, off, order, pos, ws, n, None)  # noqa: E731
    assert plan(None, 8, FAKE, FAKE, FAKE, None, 0) == qnn.QNN_EINVAL
    assert plan(FAKE, 8, None, FAKE, FAKE, None, 0) == qnn.QNN_EINVAL
    assert plan(FAKE + 2, 8, FAKE, FAKE, FAKE, None, 0) == qnn.QNN_EALIGN
    assert plan(FAKE, 1 << 20, FAKE, FAKE, FAKE, None, 0) == qnn.QNN_EWORKSPACE
    assert plan(FAKE, 1 << 20, FAKE, FAKE, FAKE, FAKE, need - 1) == qnn.QNN_EWORKSPACE
    assert plan(FAKE, 1 << 20, FAKE, FAKE, FAKE, FAKE + 16, need) == qnn.QNN_EWORKSPACE


def matmul_desc(**kw):
    d = dict(experts=1, m=100, k=128, bits=4, dtype=qnn.BF16, gated=0, act=0)
    size = kw.pop("struct_size", ctypes.sizeof(qnn.MatmulDesc))
    d.update(kw)
    return qnn.MatmulDesc(size, *(d[f] for f, _ in qnn.MatmulDesc._fields_[1:]))


@pytest.mark.parametrize("kw,want", [
    (dict(), 4 * 2 * 1024 + 128 * 8),                                  # 100 rows -> 4 blocks of 32, 128 columns -> 2 of 64
    (dict(bits=16), 4 * 2 * 4096 + 128 * 8), (dict(bits=2, k=4), 4 * 512 + 128 * 8),
    (dict(gated=1, m=9), 2 * 1024 + 32 * 8),                           # 9 channels -> 2 * 8 + 2 * 8 image rows
    (dict(experts=3, bits=8, m=32, k=64), 3 * 2048 + 3 * 32 * 8),
    (dict(experts=1024, bits=16, m=1 << 14, k=1 << 14), 1024 * (1 << 28) * 2 + 1024 * (1 << 14) * 8)])
def test_image_sizes(lib, kw, want):
    assert size_of(lib.qnn_matmul_image_size, ctypes.byref(matmul_desc(**kw))) == (qnn.QNN_OK, want)


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=0), qnn.QNN_EINVAL), (dict(experts=0), qnn.QNN_EINVAL), (dict(m=0), qnn.QNN_EINVAL), (dict(k=-1), qnn.QNN_EINVAL),
    (dict(act=5), qnn.QNN_EINVAL), (dict(gated=2), qnn.QNN_EINVAL), (dict(dtype=7), qnn.QNN_EINVAL),
    (dict(bits=3), qnn.QNN_EUNSUPPORTED), (dict(bits=32), qnn.QNN_EUNSUPPORTED), (dict(dtype=qnn.F32), qnn.QNN_EUNSUPPORTED),
    (dict(experts=1025), qnn.QNN_EUNSUPPORTED), (dict(k=127), qnn.QNN_EUNSUPPORTED), (dict(bits=2, k=126), qnn.QNN_EUNSUPPORTED)])
def test_matmul_descriptor_refusals(lib, kw, status):
    assert size_of(lib.qnn_matmul_image_size, ctypes.byref(matmul_desc(**kw)))[0] == status


def test_matmul_refusals(lib):
    d = ctypes.byref(matmul_desc())
    need = size_of(lib.qnn_matmul_image_size, d)[1]
    assert lib.qnn_matmul_prepare(d, None, None, None, FAKE, need, None) == qnn.QNN_EINVAL
    assert lib.qnn_matmul_prepare(d, FAKE, None, None, FAKE, need - 1, None) == qnn.QNN_EINVAL
    assert lib.qnn_matmul_prepare(d, FAKE, None, None, FAKE + 16, need, None) == qnn.QNN_EALIGN
    assert lib.qnn_matmul_prepare(d, FAKE, FAKE + 2, None, FAKE, need, None) == qnn.QNN_EALIGN

    def run(desc=d, t=4, x=FAKE, ldx=128, res=None, ldres=100, y=FAKE, ldy=100, f32=0, image=FAKE, size=need, ws=None, n=0):
        return lib.qnn_matmul_run(desc, image, size, t, x, ldx, res, ldres, y, ldy, f32, ws, n, None)

    assert run(x=None) == qnn.QNN_EINVAL and run(y=None) == qnn.QNN_EINVAL and run(t=-1) == qnn.QNN_EINVAL
    assert run(ldx=127) == qnn.QNN_EINVAL and run(ldy=99) == qnn.QNN_EINVAL and run(f32=2) == qnn.QNN_EINVAL
    assert run(res=FAKE, ldres=99) == qnn.QNN_EINVAL and run(image=None) == qnn.QNN_EINVAL and run(size=need - 1) == qnn.QNN_EINVAL
    assert run(desc=ctypes.byref(matmul_desc(experts=2)), size=2 * need) == qnn.QNN_EINVAL  # a plain product has one matrix
    assert run(x=FAKE + 1) == qnn.QNN_EALIGN and run(f32=1, y=FAKE + 2) == qnn.QNN_EALIGN
    assert run(t=(1 << 20) + 1) == qnn.QNN_EUNSUPPORTED
    # rows that are not 16-byte aligned need a copy where the tensor cores take over
    assert run(t=500, x=FAKE + 2) == qnn.QNN_EWORKSPACE and run(t=500, ldx=129) == qnn.QNN_EWORKSPACE
    assert size_of(lib.qnn_matmul_workspace_size, d, 500, FAKE, 129) == (qnn.QNN_OK, 500 * 128 * 2)
    assert size_of(lib.qnn_matmul_workspace_size, d, 500, FAKE, 128) == (qnn.QNN_OK, 0)


def test_experts_refusals(lib):
    desc = matmul_desc(experts=4, m=96)
    d = ctypes.byref(desc)
    need = size_of(lib.qnn_matmul_image_size, d)[1]

    def dispatch(tokens=8, top=2, off=FAKE, order=FAKE, x=FAKE, ldx=128, y=FAKE, ldy=96, ws=None, n=0):
        return lib.qnn_experts_dispatch(d, FAKE, need, tokens, top, off, order, x, ldx, y, ldy, ws, n, None)

    def combine(tokens=8, top=2, off=FAKE, pos=FAKE, w=FAKE, x=FAKE, y=FAKE, res=None, ldres=96, ws=FAKE, n=1 << 30):
        return lib.qnn_experts_combine(d, FAKE, need, tokens, top, off, pos, w, x, 128, res, ldres, y, 96, ws, n, None)

    assert dispatch(off=None) == qnn.QNN_EINVAL and dispatch(order=None) == qnn.QNN_EINVAL and dispatch(top=0) == qnn.QNN_EINVAL
    assert dispatch(ldx=100) == qnn.QNN_EINVAL and dispatch(ldy=95) == qnn.QNN_EINVAL and dispatch(x=FAKE + 1) == qnn.QNN_EALIGN
    assert dispatch(tokens=1 << 20, top=2) == qnn.QNN_EUNSUPPORTED and dispatch(top=1025) == qnn.QNN_EUNSUPPORTED
    assert dispatch(tokens=500) == qnn.QNN_EWORKSPACE  # the rows in the plan's order
    assert combine(pos=None) == qnn.QNN_EINVAL and combine(w=None) == qnn.QNN_EINVAL and combine(res=FAKE, ldres=95) == qnn.QNN_EINVAL
    assert combine(w=FAKE + 2) == qnn.QNN_EALIGN and combine(ws=None, n=0) == qnn.QNN_EWORKSPACE
    st, size = size_of(lib.qnn_experts_workspace_size, d, 8, 2, 1, FAKE, 128)
    assert st == qnn.QNN_OK and size == 16 * 96 * 4 and combine(n=size - 1) == qnn.QNN_EWORKSPACE
