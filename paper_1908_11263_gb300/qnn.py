"""Python binding of libqnn (include/qnn.h): argument marshalling only.

PyTorch provides device memory and the current stream; every step of the
computation runs in the library's CUDA kernels.  There is no fallback: when the
library is missing or fails to load, every call raises.

Tensor conventions (packed Q-bit data lives in uint8 tensors whose last
dimension counts bytes):
  activations  uint8 [n, h, w, c*Q/8]    weights  int8/uint8 [m, kh, kw, c*Q/8]
  outputs      uint8 [n, oh, ow, m*Q/8]

Tensors and streams are the current device's; others are refused, and so are tensors that require a gradient outside
torch.no_grad() and torch.inference_mode().  `stream` (a torch.cuda.Stream) is where a call's kernels are queued; without
it, the current stream.  What a call allocates belongs to that stream, and the stream that is current at the call may use it
too, once it is ordered after the call; other streams need record_stream(), as for any tensor.  Inputs are the caller's to
keep until the stream has passed the call; only the weights that PreparedMatmul and PreparedExperts lay out may be dropped
at once.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from . import build as _build

QNN_OK, QNN_EINVAL, QNN_EUNSUPPORTED, QNN_EALIGN, QNN_ECUDA, QNN_ETIMEOUT, QNN_EWORKSPACE = range(7)
QNN_ESCRATCH = 7
NOALLOC_SCRATCH_BYTES = 2 << 20  # QNN_NOALLOC_SCRATCH_BYTES
ALGO_AUTO, ALGO_DIRECT, ALGO_TENSORCORE, ALGO_TC_WINDOW, ALGO_TC_GENERAL = 0, 1, 2, 3, 4

EXPORTED = ("qconv_hwc_workspace_size", "qconv_hwc", "qconv_hwc_prepare", "qconv_hwc_run", "qconv_hwc_algo", "qlinear", "qmaxpool", "pack_subbyte",
            "unpack_subbyte", "qnn_device_status", "qnn_status_string", "qnn_version", "qconv_hwc_noalloc",
            "qnn_selftest_wait_timeout", "qconv_hwc_thresholds", "qconv_hwc_binary", "qconv_hwc_pool2", "qconv_hwc_pool2_run",
            "qconv_hwc_mma_operand_bits", "qconv_hwc_tc_kernel", "qnn_block_norm", "qnn_route_topk",
            "qnn_expert_plan_workspace_size", "qnn_expert_plan", "qnn_matmul_image_size", "qnn_matmul_prepare",
            "qnn_matmul_workspace_size", "qnn_matmul_run", "qnn_experts_workspace_size", "qnn_experts_dispatch",
            "qnn_experts_combine")

F16, BF16, F32 = 0, 1, 2  # QNN_F16, QNN_BF16, QNN_F32
_DTYPES = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}


class QnnError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class ConvDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(f, ctypes.c_int32) for f in (
        "n", "h", "w", "c", "m", "kh", "kw", "stride_h", "stride_w", "pad_h", "pad_w", "bits", "shift", "algo")]


class NormDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(f, ctypes.c_int32) for f in (
        "kind", "dtype", "residual_dtype", "param_dtype", "post_norm", "gates", "d")] + [(f, ctypes.c_int64) for f in (
            "t", "ldx", "ldres", "ldr", "ldh")] + [("scale", ctypes.c_float), ("eps", ctypes.c_float)]


class RouteDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(f, ctypes.c_int32) for f in (
        "dtype", "experts", "k", "score", "groups", "top_groups", "group_score", "renormalise")] + [
            ("scale", ctypes.c_float), ("t", ctypes.c_int64), ("ld", ctypes.c_int64)]


class MatmulDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(f, ctypes.c_int32) for f in (
        "experts", "m", "k", "bits", "dtype", "gated", "act")]


_lock = threading.Lock()
_lib = None


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = False):
    """Load libqnn.so (building it first only when asked)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.LIB
        if not os.path.exists(path):
            if not build_if_missing:
                raise RuntimeError(f"libqnn.so is not built ({path}); run paper_1908_11263_gb300.build.build()")
            _build.build()
        lib = ctypes.CDLL(path)
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        DP = ctypes.POINTER(ConvDesc)
        lib.qconv_hwc_workspace_size.argtypes = [DP, ctypes.POINTER(SZ)]
        lib.qconv_hwc_workspace_size.restype = I32
        lib.qconv_hwc.argtypes = [DP, P, P, P, P, P, P, P, P, SZ, P]
        lib.qconv_hwc.restype = I32
        lib.qconv_hwc_pool2.argtypes = [DP, P, P, P, P, P, P, P, P, SZ, P]
        lib.qconv_hwc_pool2.restype = I32
        lib.qconv_hwc_prepare.argtypes = [DP, P, P, P, P, P, P, SZ, P]
        lib.qconv_hwc_prepare.restype = I32
        lib.qconv_hwc_run.argtypes = [DP, P, P, P, SZ, P]
        lib.qconv_hwc_run.restype = I32
        lib.qconv_hwc_pool2_run.argtypes = [DP, P, P, P, SZ, P]
        lib.qconv_hwc_pool2_run.restype = I32
        lib.qconv_hwc_algo.argtypes = [DP]
        lib.qconv_hwc_noalloc.argtypes = [DP, P, P, P, P, P, P, P, P]
        lib.qconv_hwc_thresholds.argtypes = [DP, P, P, P, P, P, SZ, P]
        lib.qconv_hwc_binary.argtypes = [DP, P, P, P, P, P]
        lib.qconv_hwc_binary.restype = I32
        lib.qconv_hwc_thresholds.restype = I32
        lib.qconv_hwc_noalloc.restype = I32
        lib.qconv_hwc_algo.restype = I32
        lib.qconv_hwc_mma_operand_bits.argtypes = [DP]
        lib.qconv_hwc_mma_operand_bits.restype = I32
        lib.qconv_hwc_tc_kernel.argtypes = [DP]
        lib.qconv_hwc_tc_kernel.restype = I32
        lib.qlinear.argtypes = [I32, I32, I32, P, P, P, P, P]
        lib.qlinear.restype = I32
        lib.qmaxpool.argtypes = [I32] * 7 + [P, P, P]
        lib.qmaxpool.restype = I32
        lib.pack_subbyte.argtypes = [P, P, I64, I32, P]
        lib.pack_subbyte.restype = I32
        lib.unpack_subbyte.argtypes = [P, P, I64, I32, I32, P]
        lib.unpack_subbyte.restype = I32
        lib.qnn_block_norm.argtypes = [ctypes.POINTER(NormDesc)] + [P] * 10
        lib.qnn_block_norm.restype = I32
        lib.qnn_route_topk.argtypes = [ctypes.POINTER(RouteDesc)] + [P] * 5
        lib.qnn_route_topk.restype = I32
        lib.qnn_expert_plan_workspace_size.argtypes = [I64, I32, ctypes.POINTER(SZ)]
        lib.qnn_expert_plan_workspace_size.restype = I32
        lib.qnn_expert_plan.argtypes = [P, I64, I32, P, P, P, P, SZ, P]
        lib.qnn_expert_plan.restype = I32
        MP = ctypes.POINTER(MatmulDesc)
        lib.qnn_matmul_image_size.argtypes = [MP, ctypes.POINTER(SZ)]
        lib.qnn_matmul_image_size.restype = I32
        lib.qnn_matmul_prepare.argtypes = [MP, P, P, P, P, SZ, P]
        lib.qnn_matmul_prepare.restype = I32
        lib.qnn_matmul_workspace_size.argtypes = [MP, I64, P, I64, ctypes.POINTER(SZ)]
        lib.qnn_matmul_workspace_size.restype = I32
        lib.qnn_matmul_run.argtypes = [MP, P, SZ, I64, P, I64, P, I64, P, I64, I32, P, SZ, P]
        lib.qnn_matmul_run.restype = I32
        lib.qnn_experts_workspace_size.argtypes = [MP, I64, I32, I32, P, I64, ctypes.POINTER(SZ)]
        lib.qnn_experts_workspace_size.restype = I32
        lib.qnn_experts_dispatch.argtypes = [MP, P, SZ, I64, I32, P, P, P, I64, P, I64, P, SZ, P]
        lib.qnn_experts_dispatch.restype = I32
        lib.qnn_experts_combine.argtypes = [MP, P, SZ, I64, I32, P, P, P, P, I64, P, I64, P, I64, P, SZ, P]
        lib.qnn_experts_combine.restype = I32
        lib.qnn_selftest_wait_timeout.argtypes = [I64, P]
        lib.qnn_selftest_wait_timeout.restype = I32
        lib.qnn_device_status.argtypes = [P]
        lib.qnn_device_status.restype = I32
        lib.qnn_status_string.argtypes = [I32]
        lib.qnn_status_string.restype = ctypes.c_char_p
        lib.qnn_version.argtypes = []
        lib.qnn_version.restype = I32
        _lib = lib
        return lib


def status_string(status: int) -> str:
    try:
        return load().qnn_status_string(int(status)).decode()
    except Exception:
        return "unknown"


def _check(status: int, what: str):
    if status != QNN_OK:
        raise QnnError(status, what)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_current(device, name):
    """The library launches on the current device and asks that one for its properties: nothing may be on another."""
    current = _current_device()
    if device.index != current:
        raise ValueError(f"{name} is on {device}, but the current device is cuda:{current}")


def _ptr(t):
    """Pointer of a tensor that is not another device's, or NULL."""
    if t is None:
        return None
    index = t.get_device()  # -1: host memory
    if index >= 0 and index != _current_device():
        _on_current(t.device, "a tensor")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    else:
        _on_current(stream.device, "stream")
    return ctypes.c_void_p(stream.cuda_stream)


# The current stream's handle without building a Stream object (three microseconds a call on the GB300 host), where
# this torch has the function.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream_of(stream, device):
    """Handle of `stream`, or of the device's current stream; `device` is the current one."""
    if stream is None:
        return _raw_stream(device.index)
    _on_current(stream.device, "stream")
    return stream.cuda_stream


def _empty(shape, dtype, device, stream):
    """Memory of the launching stream.  Where `stream` is not the current one, memory of the current stream would not do: it
    may be a block that queued work there still uses, and it would go back there when dropped, while `stream` still writes
    it.  The current stream, where the caller goes on, is noted as a second user."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _on_current(stream.device, "stream")
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream())
    return t


def _dev(t: torch.Tensor, dtype, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def conv_desc(n, h, w, c, m, kh, kw, stride=(1, 1), pad=(0, 0), bits=8, shift=0, algo=ALGO_AUTO) -> ConvDesc:
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    ph, pw = (pad, pad) if isinstance(pad, int) else pad
    return ConvDesc(ctypes.sizeof(ConvDesc), n, h, w, c, m, kh, kw, sh, sw, ph, pw, bits, shift, algo)


def workspace_size(desc: ConvDesc) -> int:
    out = ctypes.c_size_t(0)
    _check(load().qconv_hwc_workspace_size(ctypes.byref(desc), ctypes.byref(out)), "qconv_hwc_workspace_size")
    return out.value


def conv_algo(desc: ConvDesc) -> int:
    r = load().qconv_hwc_algo(ctypes.byref(desc))
    if r < 0:
        raise QnnError(-r, "qconv_hwc_algo")
    return r


def tc_kernel(desc: ConvDesc) -> int:
    """The tensor-core kernel qconv_hwc() runs for this descriptor: ALGO_TC_WINDOW or
    ALGO_TC_GENERAL (0 for the CUDA-core kernel)."""
    r = load().qconv_hwc_tc_kernel(ctypes.byref(desc))
    if r < 0:
        raise QnnError(-r, "qconv_hwc_tc_kernel")
    return r


def mma_operand_bits(desc: ConvDesc) -> int:
    """Operand width of the tensor-core MMAs for this descriptor: 16 (fp16, kind::f16),
    8 (e4m3, kind::f8f6f4) or 0 (CUDA-core kernel)."""
    r = load().qconv_hwc_mma_operand_bits(ctypes.byref(desc))
    if r < 0:
        raise QnnError(-r, "qconv_hwc_mma_operand_bits")
    return r


def _workspace(nbytes: int, device, stream):
    """A workspace for one call.  Each call has its own: calls that several host threads make on one stream interleave
    their launches, and hold data in the workspace between them.  It is allocated on the launching stream, so it may go
    back to the allocator as soon as the call has returned; in a stream capture it comes from the graph's own memory."""
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _run_with_workspace(call, size, device, stream):
    """call(pointer, bytes, stream handle), without a workspace first (most calls need none; the library queues nothing
    where it says that one is missing), then with one of this call's own."""
    handle = _stream_of(stream, device)
    st = call(None, 0, handle)
    if st == QNN_EWORKSPACE:
        need = size()
        ws = _workspace(need, device, stream)
        st = call(ws.data_ptr(), need, handle)
    return st


def _run_conv(name, desc, tensors, workspace, stream):
    """name(desc, *tensors, workspace, bytes, stream) with the caller's workspace, or one of its own where it needs one."""
    call, device = getattr(load(), name), tensors[0].device
    d, pointers = ctypes.byref(desc), [_ptr(t) for t in tensors]
    if workspace is None:
        st = _run_with_workspace(lambda ws, n, handle: call(d, *pointers, ws, n, handle), lambda: workspace_size(desc), device, stream)
    else:
        nbytes = workspace_size(desc)
        if workspace.numel() < nbytes:
            raise ValueError("workspace too small")
        st = call(d, *pointers, _ptr(workspace), nbytes, _stream_of(stream, device))
    _check(st, name)


def conv_hwc(x, w, kappa, lam, *, bias=None, shifts=None, shift=0, bits=8, stride=1, pad=0, algo=ALGO_AUTO,
             out=None, workspace=None, stream=None):
    """Quantized HWC convolution with fused compression; returns uint8 [n, oh, ow, m*Q/8]."""
    _dev(x, torch.uint8, "x")
    _dev(w, (torch.int8, torch.uint8), "w")
    _dev(kappa, torch.int16, "kappa")
    _dev(lam, torch.int32, "lambda")
    if bias is not None:
        _dev(bias, torch.int32, "bias")
    if shifts is not None:
        _dev(shifts, torch.uint8, "shifts")
    per = 8 // bits
    n, h, wd, cb = x.shape
    m, kh, kw, cb2 = w.shape
    if cb != cb2:
        raise ValueError("x and w disagree on the channel count")
    desc = conv_desc(n, h, wd, cb * per, m, kh, kw, stride, pad, bits, shift, algo)
    oh = (h + 2 * desc.pad_h - kh) // desc.stride_h + 1
    ow = (wd + 2 * desc.pad_w - kw) // desc.stride_w + 1
    if out is None:
        out = _empty((n, oh, ow, m // per), torch.uint8, x.device, stream)
    else:
        _dev(out, torch.uint8, "out")
    _run_conv("qconv_hwc", desc, (x, w, bias, kappa, lam, shifts, out), workspace, stream)
    return out


def conv_hwc_pool2(x, w, kappa, lam, *, bias=None, shifts=None, shift=0, bits=8, pad=0, algo=ALGO_AUTO, out=None,
                   workspace=None, stream=None):
    """Quantized HWC convolution (stride 1) with fused compression and 2x2 stride-2 max-pooling
    (qconv_hwc_pool2); returns uint8 [n, oh // 2, ow // 2, m*Q/8]."""
    _dev(x, torch.uint8, "x")
    _dev(w, (torch.int8, torch.uint8), "w")
    _dev(kappa, torch.int16, "kappa")
    _dev(lam, torch.int32, "lambda")
    if bias is not None:
        _dev(bias, torch.int32, "bias")
    if shifts is not None:
        _dev(shifts, torch.uint8, "shifts")
    per = 8 // bits
    n, h, wd, cb = x.shape
    m, kh, kw, cb2 = w.shape
    if cb != cb2:
        raise ValueError("x and w disagree on the channel count")
    desc = conv_desc(n, h, wd, cb * per, m, kh, kw, 1, pad, bits, shift, algo)
    oh = h + 2 * desc.pad_h - kh + 1
    ow = wd + 2 * desc.pad_w - kw + 1
    if out is None:
        out = _empty((n, oh // 2, ow // 2, m // per), torch.uint8, x.device, stream)
    else:
        _dev(out, torch.uint8, "out")
    _run_conv("qconv_hwc_pool2", desc, (x, w, bias, kappa, lam, shifts, out), workspace, stream)
    return out


def conv_hwc_thresholds(x, w, thresholds, *, bits, stride=1, pad=0, algo=ALGO_AUTO, out=None, workspace=None,
                        stream=None):
    """Quantized HWC convolution with staircase compression (qconv_hwc_thresholds): INT-4 or INT-2
    outputs equal to the number of each channel's thresholds (int32 [m][2^Q - 1]) not above the
    accumulator; returns uint8 [n, oh, ow, m*Q/8]."""
    _dev(x, torch.uint8, "x")
    _dev(w, (torch.int8, torch.uint8), "w")
    _dev(thresholds, torch.int32, "thresholds")
    per = 8 // bits
    n, h, wd, cb = x.shape
    m, kh, kw, cb2 = w.shape
    if cb != cb2:
        raise ValueError("x and w disagree on the channel count")
    if tuple(thresholds.shape) != (m, (1 << bits) - 1):
        raise ValueError(f"thresholds must have shape {(m, (1 << bits) - 1)}")
    desc = conv_desc(n, h, wd, cb * per, m, kh, kw, stride, pad, bits, 0, algo)
    oh = (h + 2 * desc.pad_h - kh) // desc.stride_h + 1
    ow = (wd + 2 * desc.pad_w - kw) // desc.stride_w + 1
    if out is None:
        out = _empty((n, oh, ow, m // per), torch.uint8, x.device, stream)
    else:
        _dev(out, torch.uint8, "out")
    _run_conv("qconv_hwc_thresholds", desc, (x, w, thresholds, out), workspace, stream)
    return out


def conv_binary(x, w, thresholds, *, stride=1, pad=0, out=None, stream=None):
    """INT-1 convolution (qconv_hwc_binary): x uint8 [n, h, w, c/8], w uint8 [m, kh, kw, c/8] (bits,
    +1 = 1), thresholds int32 [m]; returns uint8 [n, oh, ow, m/8] output bits."""
    _dev(x, torch.uint8, "x")
    _dev(w, torch.uint8, "w")
    _dev(thresholds, torch.int32, "thresholds")
    n, h, wd, cb = x.shape
    m, kh, kw, cb2 = w.shape
    if cb != cb2:
        raise ValueError("x and w disagree on the channel count")
    desc = conv_desc(n, h, wd, cb * 8, m, kh, kw, stride, pad, 1, 0, ALGO_AUTO)
    oh = (h + 2 * desc.pad_h - kh) // desc.stride_h + 1
    ow = (wd + 2 * desc.pad_w - kw) // desc.stride_w + 1
    if out is None:
        out = _empty((n, oh, ow, m // 8), torch.uint8, x.device, stream)
    else:
        _dev(out, torch.uint8, "out")
    _check(load().qconv_hwc_binary(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(thresholds), _ptr(out), _stream(stream)),
           "qconv_hwc_binary")
    return out


def conv_hwc_noalloc(x, w, kappa, lam, out, *, bias=None, shifts=None, shift=0, bits=8, stride=1, pad=0,
                     algo=ALGO_AUTO, stream=None):
    """conv_hwc() through qconv_hwc_noalloc(): no device memory is allocated,
    neither by the library nor here (the caller passes `out`).

    For callers that cannot allocate device memory: a runtime whose memory is
    all committed to its own arenas, a latency-critical loop where an allocation
    or free would synchronise the device, a caller with no allocator to own a
    workspace.  The layer's scratch goes to the library's fixed array of
    NOALLOC_SCRATCH_BYTES per device; larger layers raise QnnError with status
    QNN_ESCRATCH.  Only descriptors that select the tensor-core kernel.  The
    first call on a device does set-up (the array's device address, the
    kernel's shared-memory limit): make it before any stream capture.  All calls
    share the array: calls on different streams must not overlap on the GPU.
    """
    _dev(x, torch.uint8, "x")
    _dev(w, (torch.int8, torch.uint8), "w")
    _dev(kappa, torch.int16, "kappa")
    _dev(lam, torch.int32, "lambda")
    _dev(out, torch.uint8, "out")
    if bias is not None:
        _dev(bias, torch.int32, "bias")
    if shifts is not None:
        _dev(shifts, torch.uint8, "shifts")
    per = 8 // bits
    n, h, wd, cb = x.shape
    m, kh, kw, cb2 = w.shape
    if cb != cb2:
        raise ValueError("x and w disagree on the channel count")
    desc = conv_desc(n, h, wd, cb * per, m, kh, kw, stride, pad, bits, shift, algo)
    oh = (h + 2 * desc.pad_h - kh) // desc.stride_h + 1
    ow = (wd + 2 * desc.pad_w - kw) // desc.stride_w + 1
    if tuple(out.shape) != (n, oh, ow, m // per):
        raise ValueError(f"out must have shape {(n, oh, ow, m // per)}, got {tuple(out.shape)}")
    st = load().qconv_hwc_noalloc(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(kappa), _ptr(lam),
                                  _ptr(shifts), _ptr(out), _stream(stream))
    _check(st, "qconv_hwc_noalloc")
    return out


class PreparedConv:
    """A layer whose filters and compression constants were prepared once
    (qconv_hwc_prepare); calling it runs only the convolution (qconv_hwc_run)."""

    def __init__(self, w, kappa, lam, *, n, h, wd, bias=None, shifts=None, shift=0, bits=8, stride=1, pad=0,
                 algo=ALGO_TENSORCORE, stream=None):
        _dev(w, (torch.int8, torch.uint8), "w")
        _dev(kappa, torch.int16, "kappa")
        _dev(lam, torch.int32, "lambda")
        per = 8 // bits
        m, kh, kw, cb = w.shape
        self.desc = conv_desc(n, h, wd, cb * per, m, kh, kw, stride, pad, bits, shift, algo)
        self.oh = (h + 2 * self.desc.pad_h - kh) // self.desc.stride_h + 1
        self.ow = (wd + 2 * self.desc.pad_w - kw) // self.desc.stride_w + 1
        self.out_shape = (n, self.oh, self.ow, m // per)
        self.nbytes = workspace_size(self.desc)
        self.workspace = _empty(max(self.nbytes, 1), torch.uint8, w.device, stream)
        self._keep = (w, kappa, lam, bias, shifts)
        st = load().qconv_hwc_prepare(ctypes.byref(self.desc), _ptr(w), _ptr(bias), _ptr(kappa), _ptr(lam),
                                      _ptr(shifts), _ptr(self.workspace), ctypes.c_size_t(self.nbytes),
                                      _stream(stream))
        _check(st, "qconv_hwc_prepare")

    def __call__(self, x, out=None, stream=None):
        _dev(x, torch.uint8, "x")
        if out is None:
            out = _empty(self.out_shape, torch.uint8, x.device, stream)
        st = load().qconv_hwc_run(ctypes.byref(self.desc), _ptr(x), _ptr(out), _ptr(self.workspace),
                                  ctypes.c_size_t(self.nbytes), _stream(stream))
        _check(st, "qconv_hwc_run")
        return out

    def pool2(self, x, out=None, stream=None):
        """The convolution with its 2x2 stride-2 max-pool fused (qconv_hwc_pool2_run); returns
        uint8 [n, oh // 2, ow // 2, m*Q/8]."""
        _dev(x, torch.uint8, "x")
        if out is None:
            n, _, _, mb = self.out_shape
            out = _empty((n, self.oh // 2, self.ow // 2, mb), torch.uint8, x.device, stream)
        st = load().qconv_hwc_pool2_run(ctypes.byref(self.desc), _ptr(x), _ptr(out), _ptr(self.workspace),
                                        ctypes.c_size_t(self.nbytes), _stream(stream))
        _check(st, "qconv_hwc_pool2_run")
        return out


def linear(x, w, bias=None, *, out=None, stream=None):
    """y[b][o] = sum_i x[b][i] * w[o][i] + bias[o]; int32 [n, m]."""
    _dev(x, torch.uint8, "x")
    _dev(w, torch.int8, "w")
    if bias is not None:
        _dev(bias, torch.int32, "bias")
    n, k = x.shape
    m, k2 = w.shape
    if k != k2:
        raise ValueError("x and w disagree on k")
    if out is None:
        out = _empty((n, m), torch.int32, x.device, stream)
    st = load().qlinear(n, k, m, _ptr(x), _ptr(w), _ptr(bias), _ptr(out), _stream(stream))
    _check(st, "qlinear")
    return out


def maxpool(x, k=2, s=2, bits=8, *, out=None, stream=None):
    """Max-pool packed NHWC activations; returns uint8 [n, oh, ow, c*Q/8]."""
    _dev(x, torch.uint8, "x")
    n, h, wd, cb = x.shape
    c = cb * 8 // bits
    oh, ow = (h - k) // s + 1, (wd - k) // s + 1
    if out is None:
        out = _empty((n, oh, ow, cb), torch.uint8, x.device, stream)
    st = load().qmaxpool(n, h, wd, c, k, s, bits, _ptr(x), _ptr(out), _stream(stream))
    _check(st, "qmaxpool")
    return out


def pack_subbyte(src, bits, *, out=None, stream=None):
    """int8 values [..., L] -> packed uint8 [..., L*Q/8] (low Q bits of each value)."""
    _dev(src, torch.int8, "src")
    shape = tuple(src.shape[:-1]) + (src.shape[-1] * bits // 8,)
    if out is None:
        out = _empty(shape, torch.uint8, src.device, stream)
    st = load().pack_subbyte(_ptr(src), _ptr(out), src.numel(), bits, _stream(stream))
    _check(st, "pack_subbyte")
    return out


def unpack_subbyte(src, bits, signed, *, out=None, stream=None):
    """packed uint8 [..., B] -> int8 [..., B*8/Q] (sign-extended when signed)."""
    _dev(src, (torch.uint8, torch.int8), "src")
    shape = tuple(src.shape[:-1]) + (src.shape[-1] * 8 // bits,)
    if out is None:
        out = _empty(shape, torch.int8, src.device, stream)
    st = load().unpack_subbyte(_ptr(src), _ptr(out), out.numel(), bits, int(bool(signed)), _stream(stream))
    _check(st, "unpack_subbyte")
    return out


# ---------------------------------------------------------------- language-model block operators

def _no_gradient(t, name):
    """The library computes no gradients: a result that a graph should hold would leave it without a word."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this library does not compute; make the call under torch.no_grad()")


def _rows(t: torch.Tensor, dtype, name, shape=None, device=None):
    """A CUDA matrix with contiguous columns and any row stride, on `device` (None: on the current one); returns (pointer,
    row stride)."""
    if t.dtype is dtype and t.is_cuda and not t.requires_grad and (
            t.get_device() == _current_device() if device is None else t.device == device):
        s = t.shape
        if len(s) == 2 and (shape is None or s == shape):
            ld, step = t.stride()
            if step == 1 and ld >= s[1]:
                return t.data_ptr(), ld
    return _rows_slow(t, dtype, name, shape, device)


def _rows_slow(t, dtype, name, shape, device):
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be a CUDA tensor" + ("" if device is None else f" on {device}"))
    if device is None:
        _on_current(t.device, name)
    _no_gradient(t, name)
    if t.dtype != dtype and not (isinstance(dtype, tuple) and t.dtype in dtype):
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name} must have shape {'[rows, columns]' if shape is None else tuple(shape)}, got {tuple(t.shape)}")
    rows, cols = t.shape
    ld = t.stride(0) if rows > 1 else max(cols, t.stride(0))
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{name} must have contiguous columns and rows that do not overlap")
    return t.data_ptr(), ld


def _param(t, dtype, name, shape, device):
    """An optional contiguous parameter; returns its pointer or None."""
    if t is None:
        return None
    if t.dtype is dtype and t.device == device and t.shape == shape and not t.requires_grad and t.is_contiguous():
        return t.data_ptr()
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape {tuple(shape)}, got {tuple(t.shape)}")
    _no_gradient(t, name)
    return t.data_ptr()


def _float_dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float16, bfloat16 or float32, got {t.dtype}")
    return code


_NORM_KINDS = {"rms": 0, "layer": 1}


def block_norm(x, residual=None, *, pre_weight=None, pre_bias=None, pre_norm=True, post_norm=False, post_weight=None,
               post_bias=None, gate=None, scale=1.0, eps=1e-6, kind="rms", residual_out=None, out=None, stream=None):
    """What stands between two blocks, in one pass (qnn_block_norm):

        u = N(x) * post_weight + post_bias if post_norm else x
        r = residual + scale * gate * u
        h = N(r) * pre_weight + pre_bias

    x [t, d]; residual [t, d] in x's dtype or float32; gate [d] or [gates, d] (t a multiple of gates, consecutive rows
    share one); weights and biases [d].  Gate, weights and biases have x's dtype, or are all float32.  Rows may be
    strided.  Returns (r, h) in the residual's and x's dtypes; with pre_norm=False only r is computed and h is None.
    residual_out may be the residual, out may be x."""
    code = _float_dtype(x, "x")
    if kind not in _NORM_KINDS:
        raise ValueError(f"kind must be 'rms' or 'layer', got {kind!r}")
    dtype = x.dtype
    px, ldx = _rows(x, dtype, "x")
    dev, shape = x.device, x.shape
    t, d = shape
    row = shape[1:]
    rdtype, pres, ldres = dtype, None, d
    if residual is not None:
        rdtype = residual.dtype
        if rdtype is not dtype and rdtype is not torch.float32:
            raise TypeError(f"residual must have x's dtype or float32, got {rdtype}")
        pres, ldres = _rows(residual, rdtype, "residual", shape, dev)
    elif residual_out is not None:
        rdtype = residual_out.dtype
        if rdtype not in (dtype, torch.float32):
            raise TypeError(f"residual_out must have x's dtype or float32, got {rdtype}")
    pdtype = dtype
    for p in (gate, post_weight, post_bias, pre_weight, pre_bias):
        if p is not None:
            pdtype = p.dtype
            if pdtype is not dtype and pdtype is not torch.float32:
                raise TypeError(f"gate, weights and biases must have x's dtype or float32, got {pdtype}")
            break
    gates, pgate = 1, None
    if gate is not None:
        if gate.dim() == 1:
            pgate = _param(gate, pdtype, "gate", row, dev)
        else:
            gates = gate.shape[0]
            if gates == 0 or t % gates:
                raise ValueError(f"{t} rows do not split evenly over {gates} gate rows")
            pgate = _param(gate, pdtype, "gate", (gates, d), dev)
    ppw, ppb = _param(post_weight, pdtype, "post_weight", row, dev), _param(post_bias, pdtype, "post_bias", row, dev)
    pw, pb = _param(pre_weight, pdtype, "pre_weight", row, dev), _param(pre_bias, pdtype, "pre_bias", row, dev)
    if residual_out is None:
        residual_out = _empty(shape, rdtype, dev, stream)
        pr, ldr = residual_out.data_ptr(), d
    else:
        pr, ldr = _rows(residual_out, rdtype, "residual_out", shape, dev)
    ph, ldh = None, d
    if not pre_norm:
        out = None
    elif out is None:
        out = _empty(shape, dtype, dev, stream)
        ph = out.data_ptr()
    else:
        ph, ldh = _rows(out, dtype, "out", shape, dev)
    desc = NormDesc(ctypes.sizeof(NormDesc), _NORM_KINDS[kind], code, _DTYPES[rdtype], _DTYPES[pdtype], int(bool(post_norm)),
                    gates, d, t, ldx, ldres, ldr, ldh, scale, eps)
    st = load().qnn_block_norm(ctypes.byref(desc), px, pres, pgate, ppw, ppb, pw, pb, pr, ph, _stream_of(stream, dev))
    _check(st, "qnn_block_norm")
    return residual_out, out


_SCORES = {"softmax": 0, "sigmoid": 1}
_GROUP_SCORES = {"max": 0, "top2": 1}


def route_topk(logits, k, *, score="softmax", bias=None, groups=1, top_groups=None, group_score="max", renormalise=True,
               scale=1.0, stream=None):
    """Each token's k experts and their weights (qnn_route_topk): logits [t, experts]; returns (weights float32 [t, k],
    ids int32 [t, k]), best first, ties to the lowest index.  The choice goes by softmax or sigmoid scores plus `bias`
    (float32 [experts]), first among `groups` when fewer than all are allowed; weights are the scores without the bias.
    Experts at -inf or NaN are closed; a token with too few open ones gets id -1 and weight 0."""
    code = _float_dtype(logits, "logits")
    if score not in _SCORES or group_score not in _GROUP_SCORES:
        raise ValueError(f"score must be 'softmax' or 'sigmoid' and group_score 'max' or 'top2', got {score!r}, {group_score!r}")
    p, ld = _rows(logits, logits.dtype, "logits")
    dev, (t, e) = logits.device, logits.shape
    pbias = _param(bias, torch.float32, "bias", (e,), dev)
    shape = (t, k if k > 0 else 0)
    weights = _empty(shape, torch.float32, dev, stream)
    ids = _empty(shape, torch.int32, dev, stream)
    desc = RouteDesc(ctypes.sizeof(RouteDesc), code, e, k, _SCORES[score], groups, groups if top_groups is None else top_groups,
                     _GROUP_SCORES[group_score], int(bool(renormalise)), scale, t, ld)
    st = load().qnn_route_topk(ctypes.byref(desc), p, pbias, weights.data_ptr(), ids.data_ptr(),
                               _stream_of(stream, dev))
    _check(st, "qnn_route_topk")
    return weights, ids


class ExpertPlan:
    """Which slots (token * top + choice) each expert serves (qnn_expert_plan): `offsets` int32 [experts + 1], `order`
    int32 [slots] (the slot at each place, -1 after the last) and `position` int32 [tokens, top] (the place of each
    slot, -1 for one that goes to no expert).  The three are views of one buffer."""

    __slots__ = ("tokens", "top", "experts", "device", "_buffer", "_offsets", "_order", "_position")

    def __init__(self, tokens, top, experts, device, stream=None):
        self.tokens, self.top, self.experts, self.device = tokens, top, experts, device
        slots = tokens * top
        self._buffer = _empty(2 * slots + experts + 1, torch.int32, device, stream)
        self._order = self._buffer.data_ptr()  # pointers
        self._position = self._order + 4 * slots
        self._offsets = self._position + 4 * slots

    @property
    def order(self):
        return self._buffer.as_strided((self.tokens * self.top,), (1,), 0)

    @property
    def position(self):
        return self._buffer.as_strided((self.tokens, self.top), (self.top, 1), self.tokens * self.top)

    @property
    def offsets(self):
        return self._buffer.as_strided((self.experts + 1,), (1,), 2 * self.tokens * self.top)


def expert_plan(ids, experts, *, stream=None) -> ExpertPlan:
    """The plan of ids int32 [tokens, top] over `experts`; ids outside [0, experts) go to no expert."""
    _dev(ids, torch.int32, "ids")
    _on_current(ids.device, "ids")
    if ids.dim() != 2:
        raise ValueError(f"ids must have shape [tokens, top], got {tuple(ids.shape)}")
    if experts <= 0:
        raise QnnError(QNN_EINVAL, "qnn_expert_plan")
    lib, p, (tokens, top) = load(), ids.data_ptr(), ids.shape
    plan = ExpertPlan(tokens, top, experts, ids.device, stream)

    def size():
        need = ctypes.c_size_t(0)
        _check(lib.qnn_expert_plan_workspace_size(tokens * top, experts, ctypes.byref(need)), "qnn_expert_plan_workspace_size")
        return need.value

    st = _run_with_workspace(lambda ws, n, handle: lib.qnn_expert_plan(
        p, tokens * top, experts, plan._offsets, plan._order, plan._position, ws, n, handle), size, plan.device, stream)
    _check(st, "qnn_expert_plan")
    return plan


_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


class _Prepared:
    """Weights laid out once for the matrix-product kernels (qnn_matmul_prepare)."""

    def __init__(self, w, scale, bias, bits, dtype, gated, act, experts, stream):
        if act not in _ACTS:
            raise ValueError(f"act must be one of {sorted(_ACTS)}, got {act!r}")
        if bits == 16:
            if w.dtype not in (torch.float16, torch.bfloat16) or dtype not in (None, w.dtype):
                raise TypeError(f"16-bit weights must be float16 or bfloat16 and dtype, if given, theirs; got {w.dtype}, {dtype}")
            _dev(w, None, "w")
            _no_gradient(w, "w")
            dtype, per = w.dtype, 1
        elif bits in (8, 4, 2):
            _dev(w, (torch.uint8, torch.int8), "w")
            dtype, per = torch.bfloat16 if dtype is None else dtype, 8 // bits
            if dtype not in (torch.float16, torch.bfloat16):
                raise TypeError(f"dtype must be float16 or bfloat16, got {dtype}")
        else:
            raise QnnError(QNN_EUNSUPPORTED, "qnn_matmul_prepare")
        if w.dim() != (3 if experts else 2):
            raise ValueError(f"w must have shape {'[experts, rows, k]' if experts else '[rows, k]'}, got {tuple(w.shape)}")
        rows = w.shape[-2]
        if gated and rows % 2:
            raise ValueError("a gated product needs as many gate rows as up rows")
        self.dtype, self.device, self.experts = dtype, w.device, w.shape[0] if experts else 1
        self.m, self.k = rows // 2 if gated else rows, w.shape[-1] * per
        pw, pscale = _ptr(w), _param(scale, torch.float32, "scale", w.shape[:-1], w.device)
        pbias = _param(bias, torch.float32, "bias", w.shape[:-1], w.device)
        self.desc = MatmulDesc(ctypes.sizeof(MatmulDesc), self.experts, self.m, self.k, bits, _DTYPES[dtype], int(bool(gated)),
                               _ACTS[act])
        self._desc = ctypes.byref(self.desc)
        lib, need = load(), ctypes.c_size_t(0)
        _check(lib.qnn_matmul_image_size(self._desc, ctypes.byref(need)), "qnn_matmul_image_size")
        self.nbytes = need.value
        self.image = _empty(self.nbytes, torch.uint8, w.device, stream)
        self._image = self.image.data_ptr()
        st = lib.qnn_matmul_prepare(self._desc, pw, pscale, pbias, self.image.data_ptr(), self.nbytes, _stream(stream))
        _check(st, "qnn_matmul_prepare")
        if stream is not None:  # the caller may drop them now
            for t in (w, scale, bias):
                if t is not None:
                    t.record_stream(stream)


class PreparedMatmul(_Prepared):
    """A matrix product with its epilogue fused: y = residual + act(scale * (x w^T) + bias), or with gated=True
    residual + act(gate) * up, where w holds the gate rows and then the up rows.

    w: float16/bfloat16 [rows, k] (bits=16), or packed signed codes uint8/int8 [rows, k*bits/8] (bits 8, 4 or 2) with
    scale float32 [rows]; bias float32 [rows].  dtype: of x, residual and outputs (for 16-bit weights, theirs)."""

    def __init__(self, w, *, scale=None, bias=None, bits=16, dtype=None, gated=False, act="none", stream=None):
        super().__init__(w, scale, bias, bits, dtype, gated, act, False, stream)

    def __call__(self, x, residual=None, *, out=None, out_dtype=None, stream=None):
        """x [t, k] -> [t, m] in x's dtype, or float32 with out_dtype=torch.float32.  out may be the residual."""
        dtype, dev, m = self.dtype, self.device, self.m
        _on_current(dev, "the layer")
        px, ldx = _rows(x, dtype, "x", None, dev)
        t, k = x.shape
        if k != self.k:
            raise ValueError(f"x must have {self.k} columns, got {k}")
        pres, ldres = (None, m) if residual is None else _rows(residual, dtype, "residual", (t, m), dev)
        if out is None:
            odtype = dtype if out_dtype is None else out_dtype
            if odtype is not dtype and odtype is not torch.float32:
                raise TypeError(f"out_dtype must be {dtype} or float32, got {odtype}")
            out = _empty((t, m), odtype, dev, stream)
            po, ldo = out.data_ptr(), m
        else:
            odtype = out.dtype
            if out_dtype not in (None, odtype):
                raise TypeError(f"out has dtype {odtype}, not {out_dtype}")
            po, ldo = _rows(out, dtype if odtype is dtype else torch.float32, "out", (t, m), dev)
        lib = load()

        def size():
            need = ctypes.c_size_t(0)
            _check(lib.qnn_matmul_workspace_size(self._desc, t, px, ldx, ctypes.byref(need)), "qnn_matmul_workspace_size")
            return need.value

        wide = int(odtype is torch.float32)
        st = _run_with_workspace(lambda ws, n, handle: lib.qnn_matmul_run(
            self._desc, self._image, self.nbytes, t, px, ldx, pres, ldres, po, ldo, wide, ws, n, handle), size, dev, stream)
        _check(st, "qnn_matmul_run")
        return out


class PreparedExperts(_Prepared):
    """One weight matrix an expert, as PreparedMatmul: w [experts, rows, ...], scale and bias float32 [experts, rows]."""

    def __init__(self, w, *, scale=None, bias=None, bits=16, dtype=None, gated=False, act="none", stream=None):
        super().__init__(w, scale, bias, bits, dtype, gated, act, True, stream)

    def _check_plan(self, plan):
        _on_current(self.device, "the layer")
        if plan.experts != self.experts:
            raise ValueError(f"the plan is over {plan.experts} experts, the weights over {self.experts}")
        if plan.device != self.device:
            raise ValueError(f"the plan must be on {self.device}")

    def _run(self, call, plan, combine, px, ldx, stream):
        def size():
            need = ctypes.c_size_t(0)
            _check(load().qnn_experts_workspace_size(self._desc, plan.tokens, plan.top, combine, px, ldx, ctypes.byref(need)),
                   "qnn_experts_workspace_size")
            return need.value

        _check(_run_with_workspace(call, size, self.device, stream), "qnn_experts_combine" if combine else "qnn_experts_dispatch")

    def dispatch(self, x, plan, *, out=None, stream=None):
        """Each place's token through its expert (qnn_experts_dispatch): x [tokens, k] -> [tokens * top, m] in the
        plan's order; rows after the last place are zero."""
        self._check_plan(plan)
        tokens, top = plan.tokens, plan.top
        px, ldx = _rows(x, self.dtype, "x", (tokens, self.k), self.device)
        shape = (tokens * top, self.m)
        if out is None:
            out = _empty(shape, self.dtype, self.device, stream)
        po, ldo = _rows(out, self.dtype, "out", shape, self.device)
        lib = load()
        self._run(lambda ws, n, handle: lib.qnn_experts_dispatch(
            self._desc, self._image, self.nbytes, tokens, top, plan._offsets, plan._order, px, ldx, po, ldo, ws, n, handle),
            plan, 0, px, ldx, stream)
        return out

    def combine(self, x, plan, weights, residual=None, *, out=None, stream=None):
        """The places' rows through their experts and back to the tokens (qnn_experts_combine):
        y[t] = residual[t] + sum_j weights[t, j] * product(position[t, j]); x [tokens * top, k] -> [tokens, m]."""
        self._check_plan(plan)
        tokens, top = plan.tokens, plan.top
        px, ldx = _rows(x, self.dtype, "x", (tokens * top, self.k), self.device)
        pw = _param(weights, torch.float32, "weights", (tokens, top), self.device)
        if pw is None:
            raise ValueError("weights are needed")
        shape = (tokens, self.m)
        pres, ldres = (None, self.m) if residual is None else _rows(residual, self.dtype, "residual", shape, self.device)
        if out is None:
            out = _empty(shape, self.dtype, self.device, stream)
        po, ldo = _rows(out, self.dtype, "out", shape, self.device)
        lib = load()
        self._run(lambda ws, n, handle: lib.qnn_experts_combine(
            self._desc, self._image, self.nbytes, tokens, top, plan._offsets, plan._position, pw, px, ldx, pres, ldres, po,
            ldo, ws, n, handle), plan, 1, px, ldx, stream)
        return out


def selftest_wait_timeout(limit_cycles: int, stream=None):
    """Enqueue the bounded-wait failure self-test (see qnn_selftest_wait_timeout)."""
    _check(load().qnn_selftest_wait_timeout(int(limit_cycles), _stream(stream)), "qnn_selftest_wait_timeout")


def device_status(stream=None):
    """Synchronise and raise if a bounded device-side wait gave up since the last check."""
    _check(load().qnn_device_status(_stream(stream)), "device status")
