"""The attention operators without a GPU: struct layouts, frequencies, the refusals that come before any CUDA call (the
pointers are never read), and the binding's own checks on tensors without memory."""
import ctypes
import math
import os
import shutil
import subprocess
from fractions import Fraction

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from attention_util import frequencies
from paper_1908_11263_gb300 import build as qbuild
from paper_1908_11263_gb300 import qnn
from test_device_refusals import Untouched

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # 256-byte aligned, never read
BF, F16, F32, I32, I64 = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.int64
OK, EINVAL, EUNSUP, EALIGN, EWORK = qnn.QNN_OK, qnn.QNN_EINVAL, qnn.QNN_EUNSUPPORTED, qnn.QNN_EALIGN, qnn.QNN_EWORKSPACE


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    return qnn.load()


STRUCTS = (("qnn_rope_scaling", qnn.RopeScaling), ("qnn_rope_desc", qnn.RopeDesc), ("qnn_cache_desc", qnn.CacheDesc),
           ("qnn_batch_desc", qnn.BatchDesc), ("qnn_append_desc", qnn.AppendDesc), ("qnn_attention_desc", qnn.AttentionDesc))


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src, lines, want = tmp_path / "sizes.c", [], []
    for struct, cls in STRUCTS:
        lines.append(f'printf("%zu ", sizeof({struct}));')
        want.append(ctypes.sizeof(cls))
        lines += [f'printf("%zu ", offsetof({struct}, {f}));' for f, _ in cls._fields_]
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    src.write_text('#include <stdio.h>\n#include "qnn.h"\nint main(void) {' + "\n".join(lines) + "return 0;}\n")
    exe = tmp_path / "sizes"
    subprocess.run([cc, "-std=c99", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
    assert [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def make(cls, defaults, kw):
    d = dict(defaults)
    size = kw.pop("struct_size", ctypes.sizeof(cls))
    d.update(kw)
    return cls(size, *(d[f] for f, _ in cls._fields_[1:]))


# ---------------------------------------------------------------- frequencies

SCALING = dict(dim=128, scaling=0, context=0, base=10000.0, factor=1.0, low=1.0, high=32.0)


@pytest.mark.parametrize("dim", [2, 10, 64, 128, 1024])
@pytest.mark.parametrize("name,kind", [("none", 0), ("linear", 1), ("base", 2), ("ramp", 3)])
def test_turns(lib, dim, name, kind):
    if dim == 2 and name == "base":
        pytest.skip("the exponent dim / (dim - 2) does not exist")
    kw = dict(base=500000.0, factor=8.0, context=8192, low=1.0, high=4.0)
    turns = (ctypes.c_uint64 * (dim // 2))()
    assert lib.qnn_rope_turns(ctypes.byref(make(qnn.RopeScaling, SCALING, dict(dim=dim, scaling=kind, **kw))), turns) == OK
    for t, f in zip(turns, frequencies(dim, scaling=name, **kw)):
        # powers, divisions and products in 64 bits: 16 roundings of 2^-53, and the last bit of the fraction
        assert abs(t / 2.0 ** 64 - f / (2 * math.pi)) <= 2.0 ** -49 * f / (2 * math.pi) + 2.0 ** -64


def test_turns_are_exact_at_far_positions(lib):
    """What the fraction leaves of an angle at position 10^9 is below 2^-20 of a turn."""
    turns = (ctypes.c_uint64 * 64)()
    assert lib.qnn_rope_turns(ctypes.byref(make(qnn.RopeScaling, SCALING, {})), turns) == OK
    p, two_pi = 10 ** 9, Fraction(31415926535897932384626433832795028841971693993751, 5 * 10 ** 48)
    for t, f in zip(turns, frequencies(128)):
        off = abs((Fraction(p * t, 1 << 64) - p * Fraction(f) / two_pi))
        assert off < Fraction(1, 1 << 20)


@pytest.mark.parametrize("kw", [dict(struct_size=4), dict(dim=0), dict(dim=7), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
                                dict(base=math.nan), dict(base=math.inf), dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.nan),
                                dict(scaling=3, factor=8.0), dict(scaling=3, factor=8.0, context=100, low=4.0, high=4.0),
                                dict(scaling=2, factor=2.0, dim=2), dict(scaling=3, factor=8.0, context=100, high=math.inf)])
def test_turns_refusals(lib, kw):
    turns = (ctypes.c_uint64 * 64)()
    assert lib.qnn_rope_turns(ctypes.byref(make(qnn.RopeScaling, SCALING, dict(kw))), turns) == EINVAL
    assert lib.qnn_rope_turns(ctypes.byref(make(qnn.RopeScaling, SCALING, {})), None) == EINVAL
    assert lib.qnn_rope_turns(None, turns) == EINVAL


# ---------------------------------------------------------------- the C entry points

ROPE = dict(dtype=qnn.BF16, heads=4, head_dim=64, dim=64, interleaved=0, wide=1, amplitude=1.0, t=8, ldx=256, hx=64, ldy=256, hy=64)


@pytest.mark.parametrize("kw,args,status", [
    (dict(struct_size=4), {}, EINVAL), (dict(dtype=3), {}, EINVAL), (dict(t=-1), {}, EINVAL), (dict(heads=0), {}, EINVAL),
    (dict(dim=63), {}, EINVAL), (dict(dim=66), {}, EINVAL), (dict(dim=-2), {}, EINVAL), (dict(interleaved=2), {}, EINVAL),
    (dict(wide=-1), {}, EINVAL), (dict(amplitude=math.inf), {}, EINVAL), (dict(ldx=-1), {}, EINVAL), (dict(ldy=255), {}, EINVAL),
    (dict(hy=63), {}, EINVAL), (dict(hy=0), {}, EINVAL), ({}, dict(x=None), EINVAL), ({}, dict(y=None), EINVAL),
    ({}, dict(positions=None), EINVAL), ({}, dict(turns=None), EINVAL), (dict(hx=1 << 41), {}, EINVAL),
    (dict(head_dim=1026, dim=64, hy=1026, ldy=8192), {}, EUNSUP), (dict(t=1 << 30), {}, EUNSUP),
    ({}, dict(x=FAKE + 1), EALIGN), (dict(dtype=qnn.F32), dict(y=FAKE + 2), EALIGN), ({}, dict(positions=FAKE + 4), EALIGN),
    (dict(wide=0), dict(positions=FAKE + 2), EALIGN), ({}, dict(turns=FAKE + 4), EALIGN)])
def test_rope_refusals(lib, kw, args, status):
    a = dict(turns=FAKE, positions=FAKE, x=FAKE, y=FAKE)
    a.update(args)
    assert lib.qnn_rope(ctypes.byref(make(qnn.RopeDesc, ROPE, dict(kw))), a["turns"], a["positions"], a["x"], a["y"], None) == status


CACHE = dict(dtype=qnn.BF16, kv_heads=2, head_dim=64, page_size=16, pages=100, k_page=2048, k_head=1024, k_row=64, v_page=2048,
             v_head=1024, v_row=64)
BATCH = dict(seqs=3, width=8, ragged=1, t=30, ldt=8)
APPEND = dict(heads=8, dim=64, interleaved=0, wide=0, amplitude=1.0, ldk=128, hk=64, ldv=128, hv=64, ldq=512, hq=64, ldo=512, ho=64)
ATTEND = dict(heads=8, causal=1, window=0, scale=0.125, q_seq=0, ldq=512, hq=64, o_seq=0, ldo=512, ho=64)

SHARED = [  # of the cache and of the batch
    (dict(struct_size=4), {}, EINVAL), (dict(dtype=5), {}, EINVAL), (dict(kv_heads=0), {}, EINVAL), (dict(page_size=0), {}, EINVAL),
    (dict(pages=-1), {}, EINVAL), (dict(k_row=-8), {}, EINVAL), (dict(dtype=qnn.F32), {}, EUNSUP), (dict(k_page=2049), {}, EALIGN),
    (dict(v_page=2052), {}, EALIGN), (dict(page_size=(1 << 30) + 1, k_page=1 << 40, v_page=1 << 40, kv_heads=1), {}, EUNSUP),
    ({}, dict(struct_size=4), EINVAL), ({}, dict(seqs=-1), EINVAL), ({}, dict(width=-1), EINVAL), ({}, dict(t=-1), EINVAL),
    ({}, dict(ragged=2), EINVAL), ({}, dict(ldt=-1), EINVAL), ({}, dict(ragged=0, t=31), EINVAL), ({}, dict(width=1 << 27), EUNSUP),
    ({}, dict(t=1 << 31), EUNSUP)]


def append(lib, cache=None, batch=None, desc=None, **args):
    a = dict(table=FAKE, lengths=FAKE, offsets=FAKE, turns=FAKE, positions=None, k=FAKE, v=FAKE, q=FAKE, k_pages=FAKE, v_pages=FAKE,
             q_out=FAKE)
    a.update(args)
    return lib.qnn_cache_append(ctypes.byref(make(qnn.CacheDesc, CACHE, dict(cache or {}))),
                                ctypes.byref(make(qnn.BatchDesc, BATCH, dict(batch or {}))),
                                ctypes.byref(make(qnn.AppendDesc, APPEND, dict(desc or {}))), *a.values(), None)


@pytest.mark.parametrize("cache,batch,status", SHARED + [
    (dict(k_head=1016), {}, EINVAL), (dict(v_row=56), {}, EINVAL), (dict(k_page=0), {}, EINVAL)])
def test_append_shared_refusals(lib, cache, batch, status):
    assert append(lib, cache, batch) == status


@pytest.mark.parametrize("desc,args,status", [
    (dict(struct_size=4), {}, EINVAL), (dict(heads=-1), {}, EINVAL), (dict(dim=66), {}, EINVAL), (dict(dim=3), {}, EINVAL),
    (dict(interleaved=3), {}, EINVAL), (dict(amplitude=math.nan), {}, EINVAL), (dict(ldo=500), {}, EINVAL), (dict(ldk=-1), {}, EINVAL),
    ({}, dict(k=None), EINVAL), ({}, dict(v=None), EINVAL), ({}, dict(q=None), EINVAL), ({}, dict(q_out=None), EINVAL),
    ({}, dict(k_pages=None), EINVAL), ({}, dict(table=None), EINVAL), ({}, dict(lengths=None), EINVAL), ({}, dict(offsets=None), EINVAL),
    ({}, dict(turns=None), EINVAL), (dict(heads=1 << 27, ho=64, ldo=1 << 33), {}, EUNSUP), ({}, dict(k_pages=FAKE + 8), EALIGN),
    ({}, dict(v_pages=FAKE + 2), EALIGN), ({}, dict(q=FAKE + 1), EALIGN), ({}, dict(table=FAKE + 2), EALIGN),
    ({}, dict(turns=FAKE + 4), EALIGN), (dict(wide=1), dict(positions=FAKE + 4), EALIGN)])
def test_append_refusals(lib, desc, args, status):
    assert append(lib, desc=desc, **args) == status


def attend(lib, cache=None, batch=None, desc=None, **args):
    a = dict(table=FAKE, lengths=FAKE, offsets=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, ws=FAKE, n=1 << 40)
    a.update(args)
    return lib.qnn_attention(ctypes.byref(make(qnn.CacheDesc, CACHE, dict(cache or {}))),
                             ctypes.byref(make(qnn.BatchDesc, BATCH, dict(batch or {}))),
                             ctypes.byref(make(qnn.AttentionDesc, ATTEND, dict(desc or {}))), *a.values(), None)


@pytest.mark.parametrize("cache,batch,status", SHARED + [
    (dict(head_dim=60), {}, EUNSUP), (dict(head_dim=264), {}, EUNSUP), (dict(kv_heads=3), {}, EINVAL), ({}, dict(t=1 << 28), EUNSUP)])
def test_attention_shared_refusals(lib, cache, batch, status):
    assert attend(lib, cache, batch) == status


@pytest.mark.parametrize("desc,args,status", [
    (dict(struct_size=4), {}, EINVAL), (dict(heads=0), {}, EINVAL), (dict(heads=7), {}, EINVAL), (dict(causal=2), {}, EINVAL),
    (dict(window=-1), {}, EINVAL), (dict(scale=0.0), {}, EINVAL), (dict(scale=math.nan), {}, EINVAL), (dict(scale=math.inf), {}, EINVAL), (dict(scale=1e-39), {}, EINVAL),
    (dict(scale=3e38), {}, EINVAL),
    (dict(ldo=511), {}, EINVAL), (dict(ho=0), {}, EINVAL), (dict(ldq=-1), {}, EINVAL), ({}, dict(q=None), EINVAL),
    ({}, dict(out=None), EINVAL), ({}, dict(k=None), EINVAL), ({}, dict(table=None), EINVAL), ({}, dict(offsets=None), EINVAL),
    ({}, dict(k=FAKE + 8), EALIGN), ({}, dict(v=FAKE + 2), EALIGN), ({}, dict(q=FAKE + 1), EALIGN), ({}, dict(out=FAKE + 1), EALIGN),
    ({}, dict(lse=FAKE + 2), EALIGN), ({}, dict(table=FAKE + 1), EALIGN), ({}, dict(lengths=FAKE + 2), EALIGN)])
def test_attention_refusals(lib, desc, args, status):
    assert attend(lib, desc=desc, **args) == status


# ---------------------------------------------------------------- the binding

@pytest.fixture
def new(monkeypatch):
    """cuda:0 is current; returns what makes tensors, on another device with at=1."""
    monkeypatch.setattr(qnn, "_current_device", lambda: 0)
    monkeypatch.setattr(qnn, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(qnn, "_lib", Untouched())
    with FakeTensorMode():
        yield lambda *shape, dtype=BF, at=0: torch.empty(shape, dtype=dtype, device=f"cuda:{at}")


def rotary(new, dim=64, at=0):
    r = object.__new__(qnn.Rotary)
    r.dim, r.interleaved, r.amplitude = dim, 0, 1.0
    r.turns = new(dim // 2, dtype=I64, at=at)
    r.device = r.turns.device
    return r


def calls(new, at=0, **kw):
    """Every entry point; kw replaces arguments by name."""
    def cache():
        return qnn.PagedCache(kw.get("kp", new(9, 2, 16, 64, at=at)), kw.get("vp", new(9, 2, 16, 64, at=at)))

    def get(name, *shape, dtype=BF):
        return kw[name] if name in kw else new(*shape, dtype=dtype, at=at)

    t = 6
    batch = lambda: (get("table", 3, 4, dtype=I32), get("lengths", 3, dtype=I32), get("offsets", 4, dtype=I32))  # noqa: E731
    rot = lambda: kw["rotary"] if "rotary" in kw else rotary(new, at=at)  # noqa: E731
    return {
        "rope": lambda: qnn.rope(get("q", t, 8, 64), get("positions", t, dtype=I64), rot(), out=kw.get("out")),
        "append": lambda: cache().append(get("k", t, 2, 64), get("v", t, 2, 64), *batch(), rotary=rot(), q=get("q", t, 8, 64),
                                         positions=kw.get("positions"), q_out=kw.get("out")),
        "attend": lambda: cache().attend(get("q", t, 8, 64), *batch(), out=kw.get("out"), window=kw.get("window"),
                                         scale=kw.get("scale")),
        "cross": lambda: qnn.cross_attention(get("q", 3, 5, 8, 64), get("k", 3, 7, 2, 64), get("v", 3, 7, 2, 64),
                                             get("lengths", 3, dtype=I32), out=kw.get("out")),
    }


@pytest.mark.parametrize("name", ["rope", "append", "attend", "cross"])
def test_other_devices_are_refused_before_the_library(new, name):
    with pytest.raises(AssertionError, match="was reached"):
        calls(new)[name]()
    with pytest.raises(ValueError, match="cuda:1"):
        calls(new, at=1)[name]()
    side = torch.device("cuda:1")
    fields = {"rope": ("positions", "q"), "append": ("k", "v", "q", "table", "lengths", "offsets", "vp"),
              "attend": ("q", "table", "lengths", "offsets"), "cross": ("k", "v", "lengths")}[name]
    shapes = dict(positions=((6,), I64), q=((6, 8, 64), BF), k=((6, 2, 64), BF), v=((6, 2, 64), BF), table=((3, 4), I32),
                  lengths=((3,), I32), offsets=((4,), I32), vp=((9, 2, 16, 64), BF))
    if name == "cross":
        shapes.update(k=((3, 7, 2, 64), BF), v=((3, 7, 2, 64), BF))
    for f in fields:
        shape, dtype = shapes[f]
        with pytest.raises(ValueError, match="cuda:"):
            calls(new, **{f: torch.empty(shape, dtype=dtype, device=side)})[name]()
    if name in ("rope", "append"):
        with pytest.raises(ValueError, match="rotation must be on"):
            calls(new, rotary=rotary(new, at=1))[name]()


@pytest.mark.parametrize("name,field,shape", [
    ("rope", "q", (6, 8, 64)), ("rope", "out", (6, 8, 64)), ("append", "k", (6, 2, 64)), ("append", "v", (6, 2, 64)),
    ("append", "q", (6, 8, 64)), ("append", "kp", (9, 2, 16, 64)), ("append", "vp", (9, 2, 16, 64)), ("attend", "q", (6, 8, 64)),
    ("attend", "kp", (9, 2, 16, 64)), ("attend", "vp", (9, 2, 16, 64)), ("attend", "out", (6, 8, 64)), ("cross", "q", (3, 5, 8, 64)),
    ("cross", "k", (3, 7, 2, 64)), ("cross", "v", (3, 7, 2, 64))])
def test_gradients_are_refused_where_the_call_would_be_recorded(new, name, field, shape):
    t = new(*shape).requires_grad_(True)
    with pytest.raises(ValueError, match="gradient"):
        calls(new, **{field: t})[name]()
    with torch.no_grad(), pytest.raises(AssertionError, match="was reached"):
        calls(new, **{field: t})[name]()


def test_argument_checks(new):
    def refused(error, match, name, **kw):
        with pytest.raises(error, match=match):
            calls(new, **kw)[name]()

    i32 = lambda *s: new(*s, dtype=I32)  # noqa: E731
    for name in ("rope", "append", "attend", "cross"):
        bad = (3, 5, 8, 64) if name == "cross" else (6, 8, 64)
        refused((TypeError, ValueError), "dtype|float", name, q=new(*bad, dtype=torch.int8))
        refused(ValueError, "shape", name, q=new(6, 64))
        refused(ValueError, "contiguous heads", name, q=new(*bad[:-1], 128)[..., ::2])
        refused(ValueError, "CUDA tensor", name, q=torch.empty(bad, dtype=BF, device="cpu"))
    for name in ("append", "attend"):
        refused(TypeError, "int32", name, table=new(3, 4, dtype=I64))
        refused(ValueError, "shape", name, table=i32(3))
        refused(ValueError, "contiguous rows", name, table=i32(3, 8)[:, ::2])
        refused(ValueError, "shape", name, lengths=i32(4))
        refused(TypeError, "int32", name, lengths=new(3, dtype=I64))
        refused(ValueError, "shape", name, offsets=i32(3))
        refused(TypeError, "float16 or bfloat16", name, kp=new(9, 2, 16, 64, dtype=F32))
        refused(TypeError, "float16 or bfloat16", name, vp=new(9, 2, 16, 64, dtype=F32))
        refused(ValueError, "shape", name, vp=new(9, 2, 8, 64))
        refused(ValueError, "shape", name, kp=new(9, 2, 64))
        refused(ValueError, "contiguous heads", name, kp=new(9, 2, 64, 16).transpose(2, 3))
        refused(ValueError, "shape", name, out=new(6, 8, 63))
    refused(ValueError, "shape", "append", k=new(5, 2, 64))
    refused(ValueError, "shape", "append", v=new(6, 3, 64))
    refused(TypeError, "int32 or int64", "append", positions=new(6, dtype=F32))
    refused(ValueError, "shape", "rope", positions=new(5, dtype=I64))
    refused(ValueError, "takes 128 elements", "rope", rotary=rotary(new, 128))
    refused(ValueError, "takes 128 elements", "append", rotary=rotary(new, 128))
    refused(ValueError, "multiple", "attend", q=new(6, 7, 64))
    refused(ValueError, "window", "attend", window=0)
    refused(ValueError, "agree", "cross", q=new(3, 5, 7, 64))
    refused(ValueError, "agree", "cross", k=new(2, 7, 2, 64))
    refused(ValueError, "shape", "cross", v=new(3, 8, 2, 64))
    refused(ValueError, "shape", "cross", lengths=i32(2))
    cache = qnn.PagedCache(new(9, 2, 16, 64), new(9, 2, 16, 64))
    with pytest.raises(ValueError, match="evenly"):
        cache.attend(new(7, 8, 64), i32(3, 4), i32(3))
    with pytest.raises(ValueError, match="needs q"):
        cache.append(new(6, 2, 64), new(6, 2, 64), i32(3, 4), i32(3), q_out=new(6, 8, 64))
    with pytest.raises(ValueError, match="need a rotation"):
        cache.append(new(6, 2, 64), new(6, 2, 64), i32(3, 4), i32(3), positions=i32(6))


def test_sizes_past_32_bits_are_refused_not_cut(new):
    big = (1 << 32) + 4
    one = lambda *s: new(*(1 for _ in s)).expand(*s)  # noqa: E731
    for name, kw in (("rope", dict(q=one(6, big, 64))), ("append", dict(q=one(6, big, 64))), ("attend", dict(q=one(6, big, 64))),
                     ("attend", dict(kp=one(9, 2, big, 64), vp=one(9, 2, big, 64))), ("cross", dict(q=one(3, 5, big, 64))),
                     ("cross", dict(k=one(3, big, 2, 64), v=one(3, big, 2, 64)))):
        with pytest.raises(ValueError, match="2.31|contiguous heads"):
            calls(new, **kw)[name]()
    with pytest.raises(AssertionError, match="was reached"):
        calls(new, window=1 << 40)["attend"]()  # no limit


@pytest.mark.parametrize("kw,match", [
    (dict(dim=8, context=1 << 32), "2.31"), (dict(dim=7), "even"), (dict(dim=0), "even"), (dict(dim=8, scaling="half"), "scaling"), (dict(dim=8, amplitude=math.nan), "amplitude"),
    (dict(dim=8, frequencies=[1.0]), "frequencies"), (dict(dim=4, frequencies=[1.0, math.inf]), "frequencies")])
def test_rotary_checks(kw, match):
    with pytest.raises(ValueError, match=match):
        qnn.Rotary(**kw)


def test_rotary_refusals_of_the_library(lib):
    for kw in (dict(base=0.5), dict(scaling="linear", factor=0.5), dict(scaling="ramp", factor=2.0), dict(dim=2, scaling="base", factor=2.0)):
        with pytest.raises(qnn.QnnError):
            qnn.Rotary(kw.pop("dim", 8), **kw)
