"""paper_1911_07384_amd: the all-FP16 training hot path of arXiv:1911.07384
("Distributed low-precision Training Without Mixed Precision") on MI355X.

This module is a thin ctypes binding over ``libfp16train.so``, whose C ABI is
declared in ``include/fp16train.h``.  Functions carry the same names as the
C entry points and only marshal arguments: torch tensors (float16, CUDA/HIP
device, contiguous) are passed as raw device pointers, and work is enqueued
on the current torch stream unless another stream is given.  Every step of
the computation runs in the HIP kernels; there is no fallback path.  A
nonzero status raises ``Fp16Error``.
"""

from __future__ import annotations

import ctypes
import operator
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfp16train.so")

FP16_NHWC = 0
FP16_NCHW = 1
PASS_FWD, PASS_DGRAD, PASS_WGRAD = 0, 1, 2
_LAYOUTS = {"NHWC": FP16_NHWC, "NCHW": FP16_NCHW, FP16_NHWC: FP16_NHWC, FP16_NCHW: FP16_NCHW}

STATUS = {0: "FP16_OK", 1: "FP16_ERR_NULL", 2: "FP16_ERR_SHAPE", 3: "FP16_ERR_LAYOUT",
          4: "FP16_ERR_MISALIGNED", 5: "FP16_ERR_ALIASING", 6: "FP16_ERR_WORKSPACE",
          7: "FP16_ERR_UNSUPPORTED", 8: "FP16_ERR_HIP"}

EXPORTS = ["fp16_conv_out_dims", "fp16_conv_workspace_bytes", "fp16_conv_fwd", "fp16_conv_dgrad",
           "fp16_conv_dgrad_add", "fp16_conv_wgrad", "fp16_bn_workspace_bytes", "fp16_bn_relu", "fp16_bn_relu_bwd",
           "fp16_sgd_step", "fp16_pool_out_dims", "fp16_maxpool_fwd", "fp16_maxpool_bwd",
           "fp16_avgpool_fwd", "fp16_avgpool_bwd", "fp16_softmax_ce", "fp16_status_string",
           "fp16_version", "fp16_conv_bn_workspace_bytes", "fp16_conv_bn_relu_fwd",
           "fp16_sgd_step_f16", "fp16_conv_dgrad_filter_bytes", "fp16_conv_dgrad_filter",
           "fp16_conv_dgrad_filters",
           "fp16_conv_dgrad_wf", "fp16_conv_kernel", "fp16_noalloc_scratch_bytes", "fp16_conv_wgrad_noalloc",
           "fp16_bn_mask_bytes", "fp16_bn_relu_m", "fp16_bn_relu_bwd_m", "fp16_conv_bn_relu_fwd_m",
           "fp16_conv_dgrad_wf_m", "fp16_bn_relu_maxpool", "fp16_conv_wgrad_ex",
           "fp16_conv_dgrad_wf_ex", "fp16_muon_workspace_bytes", "fp16_muon_kernels", "fp16_orthogonalize",
           "fp16_muon_step", "fp16_int8_row_bytes", "fp16_int8_quant_rows",
           "fp16_int8_quant_workspace_bytes", "fp16_int8_quant_cols", "fp16_int8_matmul",
           "fp16_int8_kernel", "fp16_int8_dense_workspace_bytes", "fp16_int8_dense_weights",
           "fp16_int8_dense_fwd", "fp16_int8_dense_bwd", "fp16_rng_advance", "fp16_dropout",
           "fp16_dense_workspace_bytes", "fp16_dense_fwd", "fp16_dense_bwd", "fp16_dense_kernel",
           "fp16_logprobs_workspace_bytes", "fp16_logprobs", "fp16_logprobs_bwd"]


class Fp16Error(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {STATUS.get(status, status)} ({_status_string(status)})")


class ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n", "c", "h", "w", "k", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w",
                 "layout", "accum")]


class BnDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("c", ctypes.c_int32), ("h", ctypes.c_int32),
                ("w", ctypes.c_int32), ("layout", ctypes.c_int32), ("eps", ctypes.c_float),
                ("post_scale", ctypes.c_float), ("relu", ctypes.c_int32),
                ("use_stats", ctypes.c_int32), ("swap", ctypes.c_int32)]


class PoolDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n", "c", "h", "w", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w", "layout")]


class MuonDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("scale", ctypes.c_float)]


class Int8DenseDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "inputs", "outputs")]


class DenseDesc(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("inputs", ctypes.c_int32),
                ("outputs", ctypes.c_int32), ("act", ctypes.c_int32), ("drop", ctypes.c_float),
                ("site", ctypes.c_uint32)]


class LogprobDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("classes", ctypes.c_int32), ("stride", ctypes.c_int32),
                ("scale", ctypes.c_float), ("top", ctypes.c_int32)]


_lib = None
_P = ctypes.c_void_p
_SZ = ctypes.c_size_t
_F = ctypes.c_float
_I32 = ctypes.c_int32
_SIGS = {
    "fp16_conv_out_dims": (ctypes.c_int, [_P, _P, _P]),
    "fp16_conv_workspace_bytes": (_SZ, [_P, _I32]),
    "fp16_conv_fwd": (ctypes.c_int, [_P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_dgrad": (ctypes.c_int, [_P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_dgrad_add": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_wgrad": (ctypes.c_int, [_P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_dgrad_filter_bytes": (_SZ, [_P]),
    "fp16_noalloc_scratch_bytes": (_SZ, []),
    "fp16_conv_wgrad_noalloc": (ctypes.c_int, [_P, _P, _P, _P, _P]),
    "fp16_conv_dgrad_filter": (ctypes.c_int, [_P, _P, _P, _P]),
    "fp16_conv_dgrad_filters": (ctypes.c_int, [ctypes.c_int32, _P, _P, _P, _P]),
    "fp16_conv_dgrad_wf": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_dgrad_wf_m": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_bn_relu_maxpool": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_conv_wgrad_ex": (ctypes.c_int, [_P, _P, _P, _P, _P, _SZ, ctypes.c_int32, _P]),
    "fp16_conv_dgrad_wf_ex": (ctypes.c_int, [_P, _P, _P, _P, _P, ctypes.c_int32, _P, _P, _SZ, _P]),
    "fp16_bn_workspace_bytes": (_SZ, [_P]),
    "fp16_bn_mask_bytes": (_SZ, [_P]),
    "fp16_bn_relu_m": (ctypes.c_int, [_P] * 9 + [_SZ, _P]),
    "fp16_bn_relu_bwd_m": (ctypes.c_int, [_P] * 12 + [_SZ, _P]),
    "fp16_conv_bn_relu_fwd_m": (ctypes.c_int, [_P] * 12 + [_SZ, _P]),
    "fp16_bn_relu": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "fp16_bn_relu_bwd": (ctypes.c_int, [_P] * 13 + [_SZ, _P]),
    "fp16_sgd_step": (ctypes.c_int, [_P, _P, _P, _SZ, _F, _F, _F, _P]),
    "fp16_sgd_step_f16": (ctypes.c_int, [_P, _P, _P, _SZ, _F, _F, _F, _P]),
    "fp16_pool_out_dims": (ctypes.c_int, [_P, _P, _P]),
    "fp16_maxpool_fwd": (ctypes.c_int, [_P, _P, _P, _P, _P]),
    "fp16_maxpool_bwd": (ctypes.c_int, [_P, _P, _P, _P, _P]),
    "fp16_avgpool_fwd": (ctypes.c_int, [_P, _P, _P, _P]),
    "fp16_avgpool_bwd": (ctypes.c_int, [_P, _P, _P, _P]),
    "fp16_softmax_ce": (ctypes.c_int, [_I32, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "fp16_conv_bn_workspace_bytes": (_SZ, [_P, _P]),
    "fp16_conv_bn_relu_fwd": (ctypes.c_int, [_P] * 11 + [_SZ, _P]),
    "fp16_conv_kernel": (ctypes.c_char_p, [_P, _I32, _I32]),
    "fp16_muon_workspace_bytes": (_SZ, [_I32, _P, _I32]),
    "fp16_muon_kernels": (ctypes.c_char_p, [_I32, _P, _I32]),
    "fp16_orthogonalize": (ctypes.c_int, [_I32, _P, _P, _P, _I32, _P, _I32, _P, _SZ, _P]),
    "fp16_muon_step": (ctypes.c_int, [_I32, _P, _P, _P, _P, _F, _F, _F, _I32, _I32, _P, _I32, _P,
                                      _SZ, _P]),
    "fp16_int8_row_bytes": (_SZ, [_I32]),
    "fp16_int8_quant_rows": (ctypes.c_int, [_I32, _I32, _P, _P, _P, _P]),
    "fp16_int8_quant_workspace_bytes": (_SZ, [_I32, _I32]),
    "fp16_int8_quant_cols": (ctypes.c_int, [_I32, _I32, _P, _P, _P, _P, _SZ, _P]),
    "fp16_int8_matmul": (ctypes.c_int, [_I32] * 3 + [_P] * 7),
    "fp16_int8_kernel": (ctypes.c_char_p, [_I32] * 3),
    "fp16_int8_dense_workspace_bytes": (_SZ, [_P, _I32]),
    "fp16_int8_dense_weights": (ctypes.c_int, [_P] * 7 + [_SZ, _P]),
    "fp16_int8_dense_fwd": (ctypes.c_int, [_P] * 7 + [_SZ, _P]),
    "fp16_int8_dense_bwd": (ctypes.c_int, [_P] * 9 + [_SZ, _P]),
    "fp16_rng_advance": (ctypes.c_int, [_P, ctypes.c_uint64, _P]),
    "fp16_dropout": (ctypes.c_int, [_SZ, _P, _P, _P, _F, _P, ctypes.c_uint32, _P]),
    "fp16_dense_workspace_bytes": (_SZ, [_P, _I32]),
    "fp16_dense_fwd": (ctypes.c_int, [_P] * 9 + [_SZ, _P]),
    "fp16_dense_bwd": (ctypes.c_int, [_P] * 10 + [_SZ, _P]),
    "fp16_dense_kernel": (ctypes.c_char_p, [_P, _I32]),
    "fp16_logprobs_workspace_bytes": (_SZ, [_P]),
    "fp16_logprobs": (ctypes.c_int, [_P] * 8 + [_SZ, _P]),
    "fp16_logprobs_bwd": (ctypes.c_int, [_P] * 8),
    "fp16_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "fp16_version": (ctypes.c_char_p, []),
}


def lib() -> ctypes.CDLL:
    """The loaded HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -c 'import "
                               f"__graft_entry__ as g; g.build()'` (no fallback path exists)")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(l, name)
            f.restype = res
            f.argtypes = args
        _lib = l
    return _lib


def _status_string(status: int) -> str:
    try:
        return lib().fp16_status_string(int(status)).decode()
    except Exception:  # pragma: no cover - only when the library cannot load
        return "?"


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise Fp16Error(fn, status)


_DTYPES = frozenset()  # the element types a buffer may have (filled at first use)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if t.dtype not in _DTYPES:
        _check_dtype(t)
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _check_dtype(t) -> None:
    global _DTYPES
    import torch
    _DTYPES = frozenset((torch.float16, torch.float32, torch.uint8, torch.int32))
    if t.dtype not in _DTYPES:
        raise TypeError(f"expected float16/float32/uint8/int32 tensor, got {t.dtype}")


def _ptr_of(dtype):
    """A _ptr for arguments of one element type, named as in torch."""
    want = None

    def ptr(t):
        nonlocal want
        if t is None or isinstance(t, int):
            return t
        if t.dtype is not want:
            import torch
            want = getattr(torch, dtype)
            if t.dtype is not want:
                raise TypeError(f"expected {dtype} tensor, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return t.data_ptr()
    return ptr


_ptr_half, _ptr_float, _ptr_int8 = _ptr_of("float16"), _ptr_of("float32"), _ptr_of("int8")


def _held_of(dtype):
    """A _ptr for arguments of one element type, a number of elements at least and a
    device, which `what` names."""
    want = None

    def ptr(t, n, what, device):
        nonlocal want
        if t is None or isinstance(t, int):
            return t
        if t.dtype is not want:
            import torch
            want = getattr(torch, dtype)
            if t.dtype is not want:
                raise TypeError(f"{what}: expected {dtype} tensor, got {t.dtype}")
        if t.numel() < n:
            raise ValueError(f"{what} has {t.numel()} elements of {n}")
        if t.get_device() != device:
            raise ValueError(f"{what} is on {t.device}, which is not the current device")
        if not t.is_contiguous():
            raise ValueError(f"{what}: tensor must be contiguous")
        return t.data_ptr()
    return ptr


_held_half, _held_float, _held_int, _held_long = (_held_of(d) for d in (
    "float16", "float32", "int32", "int64"))


def _first_current_stream():
    """The current stream of the current device; from the second call on asked
    of torch's C++ side directly (torch.cuda.current_stream() builds a Stream
    object, 2.8 us of the 7.9 us that a call took on the host; 4.3 us now)."""
    global _current_stream
    import torch
    s = torch.cuda.current_stream().cuda_stream  # initialises the device, or raises
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and device is not None:
        def current():
            return raw(device())
        if current() == s:
            _current_stream = current
    return s


_current_stream = _first_current_stream


def _first_device():
    """The current device (-1, a CPU tensor's, where there is none); later calls ask
    torch's C++ side as _current_stream does."""
    global _device
    import torch
    if not torch.cuda.is_available():
        return -1
    d = torch.cuda.current_device()
    raw = getattr(torch._C, "_cuda_getDevice", None)
    if raw is not None and raw() == d:
        _device = raw
    return d


_device = _first_device


def _held_ws(ws, ws_bytes, device):
    """A workspace's address and bytes, at most a tensor's own."""
    if ws is None or isinstance(ws, int):
        size = 0 if ws_bytes is None else int(ws_bytes)
        if size < 0:
            raise ValueError(f"ws_bytes {size}")
        return ws, size
    if ws.get_device() != device:
        raise ValueError(f"ws is on {ws.device}, which is not the current device")
    if not ws.is_contiguous():
        raise ValueError("ws: tensor must be contiguous")
    size = ws.nbytes
    if ws_bytes is not None:
        if not 0 <= ws_bytes <= size:
            raise ValueError(f"ws has {size} bytes, ws_bytes is {ws_bytes}")
        size = int(ws_bytes)
    return ws.data_ptr(), size


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def conv_desc(n, c, h, w, k, r, s, stride=1, pad=0, layout="NHWC", accum=0) -> ConvDesc:
    """accum = 1 selects binary16 accumulation (see fp16_conv_desc.accum)."""
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    ph, pw = (pad, pad) if isinstance(pad, int) else pad
    return ConvDesc(n, c, h, w, k, r, s, sh, sw, ph, pw, _LAYOUTS[layout], int(accum))


def bn_desc(n, c, h, w, layout="NHWC", eps=1e-5, post_scale=1.0, relu=True, use_stats=False,
            swap=False) -> BnDesc:
    return BnDesc(n, c, h, w, _LAYOUTS[layout], eps, post_scale, int(bool(relu)),
                  int(bool(use_stats)), int(bool(swap)))


# ---- C entry points, same names --------------------------------------------

def fp16_version() -> str:
    return lib().fp16_version().decode()


def fp16_status_string(status: int) -> str:
    return lib().fp16_status_string(int(status)).decode()


def fp16_conv_out_dims(desc: ConvDesc):
    p, q = ctypes.c_int32(), ctypes.c_int32()
    _check("fp16_conv_out_dims", lib().fp16_conv_out_dims(ctypes.byref(desc), ctypes.byref(p),
                                                          ctypes.byref(q)))
    return p.value, q.value


def fp16_conv_kernel(desc: ConvDesc, pass_: int, addend: bool = False, stats: bool = False) -> str:
    """The kernel a pass runs on and its tile (for tests and profiles)."""
    return lib().fp16_conv_kernel(ctypes.byref(desc), int(pass_),
                                  int(addend) + 2 * int(stats)).decode()


def fp16_conv_workspace_bytes(desc: ConvDesc, pass_: int) -> int:
    return int(lib().fp16_conv_workspace_bytes(ctypes.byref(desc), int(pass_)))


def fp16_conv_fwd(desc, x, w, y, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_fwd", lib().fp16_conv_fwd(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(y),
                                                _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_dgrad(desc, dy, w, dx, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_dgrad", lib().fp16_conv_dgrad(ctypes.byref(desc), _ptr(dy), _ptr(w), _ptr(dx),
                                                    _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_dgrad_add(desc, dy, w, addend, dx, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_dgrad_add", lib().fp16_conv_dgrad_add(
        ctypes.byref(desc), _ptr(dy), _ptr(w), _ptr(addend), _ptr(dx), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


def fp16_conv_dgrad_filter_bytes(desc: ConvDesc) -> int:
    return int(lib().fp16_conv_dgrad_filter_bytes(ctypes.byref(desc)))


def fp16_conv_dgrad_filter(desc, w, wf, stream=None) -> None:
    _check("fp16_conv_dgrad_filter", lib().fp16_conv_dgrad_filter(ctypes.byref(desc), _ptr(w),
                                                                  _ptr(wf), _stream(stream)))


def fp16_conv_dgrad_filters(descs, ws, wfs, stream=None) -> None:
    """fp16_conv_dgrad_filter for every (desc, w, wf) of the three lists."""
    n = len(descs)
    if not (len(ws) == len(wfs) == n):
        raise ValueError("descs, ws and wfs differ in length")
    d = (ConvDesc * max(n, 1))(*descs)
    w = (ctypes.c_void_p * max(n, 1))(*[_ptr(t) for t in ws])
    f = (ctypes.c_void_p * max(n, 1))(*[_ptr(t) for t in wfs])
    _check("fp16_conv_dgrad_filters", lib().fp16_conv_dgrad_filters(n, d, w, f, _stream(stream)))


def fp16_conv_dgrad_wf(desc, dy, wf, addend, dx, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_dgrad_wf", lib().fp16_conv_dgrad_wf(
        ctypes.byref(desc), _ptr(dy), _ptr(wf), _ptr(addend), _ptr(dx), _ptr(ws),
        _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_dgrad_wf_m(desc, dy, wf, addend, mask, dx, ws=None, ws_bytes=None,
                         stream=None) -> None:
    _check("fp16_conv_dgrad_wf_m", lib().fp16_conv_dgrad_wf_m(
        ctypes.byref(desc), _ptr(dy), _ptr(wf), _ptr(addend), _ptr(mask), _ptr(dx), _ptr(ws),
        _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_dgrad_wf_ex(desc, dy, wf, addend, mask, addend_stride, dx, ws=None, ws_bytes=None,
                          stream=None) -> None:
    _check("fp16_conv_dgrad_wf_ex", lib().fp16_conv_dgrad_wf_ex(
        ctypes.byref(desc), _ptr(dy), _ptr(wf), _ptr(addend), _ptr(mask), int(addend_stride),
        _ptr(dx), _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_wgrad(desc, x, dy, dw, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_wgrad", lib().fp16_conv_wgrad(ctypes.byref(desc), _ptr(x), _ptr(dy), _ptr(dw),
                                                    _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_conv_wgrad_ex(desc, x, dy, dw, ws=None, ws_bytes=None, workgroups=0,
                       stream=None) -> None:
    _check("fp16_conv_wgrad_ex", lib().fp16_conv_wgrad_ex(
        ctypes.byref(desc), _ptr(x), _ptr(dy), _ptr(dw), _ptr(ws), _wsb(ws, ws_bytes),
        int(workgroups), _stream(stream)))


def fp16_noalloc_scratch_bytes() -> int:
    return int(lib().fp16_noalloc_scratch_bytes())


def fp16_conv_wgrad_noalloc(desc, x, dy, dw, stream=None) -> None:
    _check("fp16_conv_wgrad_noalloc", lib().fp16_conv_wgrad_noalloc(
        ctypes.byref(desc), _ptr(x), _ptr(dy), _ptr(dw), _stream(stream)))


def fp16_bn_workspace_bytes(desc: BnDesc) -> int:
    return int(lib().fp16_bn_workspace_bytes(ctypes.byref(desc)))


def fp16_bn_relu(desc, x, gamma, beta, residual, y, stats, ws=None, ws_bytes=None,
                 stream=None) -> None:
    _check("fp16_bn_relu", lib().fp16_bn_relu(ctypes.byref(desc), _ptr(x), _ptr(gamma), _ptr(beta),
                                              _ptr(residual), _ptr(y), _ptr(stats), _ptr(ws),
                                              _wsb(ws, ws_bytes), _stream(stream)))


def fp16_bn_relu_bwd(desc, x, y, dy, gamma, beta, residual, stats, dx, dgamma, dbeta, dresidual,
                     ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_bn_relu_bwd", lib().fp16_bn_relu_bwd(
        ctypes.byref(desc), _ptr(x), _ptr(y), _ptr(dy), _ptr(gamma), _ptr(beta), _ptr(residual),
        _ptr(stats), _ptr(dx), _ptr(dgamma), _ptr(dbeta), _ptr(dresidual), _ptr(ws),
        _wsb(ws, ws_bytes), _stream(stream)))


def fp16_bn_mask_bytes(desc: BnDesc) -> int:
    return int(lib().fp16_bn_mask_bytes(ctypes.byref(desc)))


def fp16_bn_relu_m(desc, x, gamma, beta, residual, y, stats, mask, ws=None, ws_bytes=None,
                   stream=None) -> None:
    _check("fp16_bn_relu_m", lib().fp16_bn_relu_m(
        ctypes.byref(desc), _ptr(x), _ptr(gamma), _ptr(beta), _ptr(residual), _ptr(y), _ptr(stats),
        _ptr(mask), _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_bn_relu_bwd_m(desc, x, mask, dy, gamma, beta, stats, dx, dgamma, dbeta, dresidual,
                       ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_bn_relu_bwd_m", lib().fp16_bn_relu_bwd_m(
        ctypes.byref(desc), _ptr(x), _ptr(mask), _ptr(dy), _ptr(gamma), _ptr(beta), _ptr(stats),
        _ptr(dx), _ptr(dgamma), _ptr(dbeta), _ptr(dresidual), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


def fp16_sgd_step(w, g, m, n=None, lr=0.1, momentum=0.9, weight_decay=1e-4, stream=None) -> None:
    if n is None:
        n = w.numel()
    _check("fp16_sgd_step", lib().fp16_sgd_step(_ptr(w), _ptr(g), _ptr(m), int(n), float(lr),
                                                float(momentum), float(weight_decay),
                                                _stream(stream)))


def fp16_sgd_step_f16(w, g, m, n=None, lr=0.1, momentum=0.9, weight_decay=1e-4,
                      stream=None) -> None:
    if n is None:
        n = w.numel()
    _check("fp16_sgd_step_f16", lib().fp16_sgd_step_f16(_ptr(w), _ptr(g), _ptr(m), int(n),
                                                        float(lr), float(momentum),
                                                        float(weight_decay), _stream(stream)))


def pool_desc(n, c, h, w, r, s, stride=1, pad=0, layout="NHWC") -> PoolDesc:
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    ph, pw = (pad, pad) if isinstance(pad, int) else pad
    return PoolDesc(n, c, h, w, r, s, sh, sw, ph, pw, _LAYOUTS[layout])


def fp16_pool_out_dims(desc: PoolDesc):
    p, q = ctypes.c_int32(), ctypes.c_int32()
    _check("fp16_pool_out_dims", lib().fp16_pool_out_dims(ctypes.byref(desc), ctypes.byref(p),
                                                          ctypes.byref(q)))
    return p.value, q.value


def fp16_maxpool_fwd(desc, x, y, idx, stream=None) -> None:
    _check("fp16_maxpool_fwd", lib().fp16_maxpool_fwd(ctypes.byref(desc), _ptr(x), _ptr(y),
                                                      _ptr(idx), _stream(stream)))


def fp16_bn_relu_maxpool(bn, pool, x, gamma, beta, stats, y, idx, ws=None, ws_bytes=None,
                         stream=None) -> None:
    _check("fp16_bn_relu_maxpool", lib().fp16_bn_relu_maxpool(
        ctypes.byref(bn), ctypes.byref(pool), _ptr(x), _ptr(gamma), _ptr(beta), _ptr(stats),
        _ptr(y), _ptr(idx), _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_maxpool_bwd(desc, idx, dy, dx, stream=None) -> None:
    _check("fp16_maxpool_bwd", lib().fp16_maxpool_bwd(ctypes.byref(desc), _ptr(idx), _ptr(dy),
                                                      _ptr(dx), _stream(stream)))


def fp16_avgpool_fwd(desc, x, y, stream=None) -> None:
    _check("fp16_avgpool_fwd", lib().fp16_avgpool_fwd(ctypes.byref(desc), _ptr(x), _ptr(y),
                                                      _stream(stream)))


def fp16_avgpool_bwd(desc, dy, dx, stream=None) -> None:
    _check("fp16_avgpool_bwd", lib().fp16_avgpool_bwd(ctypes.byref(desc), _ptr(dy), _ptr(dx),
                                                      _stream(stream)))


def fp16_softmax_ce(n, k, z, bias, labels, loss, dz, dbias, stream=None) -> None:
    _check("fp16_softmax_ce", lib().fp16_softmax_ce(int(n), int(k), _ptr(z), _ptr(bias),
                                                    _ptr(labels), _ptr(loss), _ptr(dz),
                                                    _ptr(dbias), _stream(stream)))


def fp16_conv_bn_workspace_bytes(conv: ConvDesc, bn: BnDesc) -> int:
    return int(lib().fp16_conv_bn_workspace_bytes(ctypes.byref(conv), ctypes.byref(bn)))


def fp16_conv_bn_relu_fwd(conv, bn, x, w, gamma, beta, residual, y, z, stats, ws=None,
                          ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_bn_relu_fwd", lib().fp16_conv_bn_relu_fwd(
        ctypes.byref(conv), ctypes.byref(bn), _ptr(x), _ptr(w), _ptr(gamma), _ptr(beta),
        _ptr(residual), _ptr(y), _ptr(z), _ptr(stats), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


def fp16_conv_bn_relu_fwd_m(conv, bn, x, w, gamma, beta, residual, y, z, stats, mask, ws=None,
                            ws_bytes=None, stream=None) -> None:
    _check("fp16_conv_bn_relu_fwd_m", lib().fp16_conv_bn_relu_fwd_m(
        ctypes.byref(conv), ctypes.byref(bn), _ptr(x), _ptr(w), _ptr(gamma), _ptr(beta),
        _ptr(residual), _ptr(y), _ptr(z), _ptr(stats), _ptr(mask), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


# ---- orthogonalised momentum ------------------------------------------------

def muon_descs(shapes):
    """The descriptors of a set of matrices: (rows, cols) or (rows, cols, scale) each."""
    return (MuonDesc * len(shapes))(*[MuonDesc(*s) if len(s) == 3 else MuonDesc(*s, 1.0)
                                      for s in shapes])


def _muon_list(descs, *lists):
    """The number of matrices and an array of pointers for each list of tensors, which
    are binary16 and of their matrices' sizes at least."""
    n = len(lists[0])
    if any(len(l) != n for l in (descs, *lists)):
        raise ValueError("descs and the lists of tensors differ in length")
    v = memoryview(descs).cast("B").cast("i").tolist()  # rows, cols and the scale's bits
    need = [r * c for r, c in zip(v[::3], v[1::3])]
    for l in lists:
        try:
            have = [t.numel() for t in l]
        except AttributeError:  # addresses among them, which are taken as they are
            have = [t.numel() if hasattr(t, "numel") else k for t, k in zip(l, need)]
        if any(map(operator.lt, have, need)):
            raise ValueError(f"matrices of {need} elements, tensors of {have}")
    return [n] + [(_P * n)(*map(_ptr_half, l)) for l in lists]


def _coef(coef, steps):
    """None, one (a, b, c) for every step, or one for each step."""
    if coef is None:
        return None
    flat = [float(v) for c in coef for v in (c if isinstance(c, (tuple, list)) else (c,))]
    if len(flat) == 3:
        flat *= int(steps)
    if len(flat) != 3 * int(steps):
        raise ValueError("coef holds (a, b, c), or steps of them")
    return (_F * max(len(flat), 1))(*flat)


def fp16_muon_workspace_bytes(descs, products=None) -> int:
    """Workspace with this many products, or (None) enough for one and for three."""
    return max(int(lib().fp16_muon_workspace_bytes(len(descs), descs, p))
               for p in ((1, 3) if products is None else (int(products),)))


def fp16_muon_kernels(descs, products=1) -> str:
    """The tiles that the products run on (for tests and profiles)."""
    return lib().fp16_muon_kernels(len(descs), descs, int(products)).decode()


def fp16_orthogonalize(descs, xs, ys, steps=5, coef=None, products=3, ws=None, ws_bytes=None,
                       stream=None) -> None:
    """Each x of xs orthogonalised into the y of ys (lists of tensors)."""
    n, x, y = _muon_list(descs, xs, ys)
    _check("fp16_orthogonalize", lib().fp16_orthogonalize(
        n, descs, x, y, int(steps), _coef(coef, steps), int(products), _ptr(ws),
        _wsb(ws, ws_bytes), _stream(stream)))


def fp16_muon_step(descs, ws_, gs, ms, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True,
                   steps=5, coef=None, products=1, ws=None, ws_bytes=None, stream=None) -> None:
    """One update of the weights ws_ from the gradients gs with the momenta ms.
    products: operands of the orthogonalisation rounded to binary16 (1) or of 22 bits
    (3), see the header for what either keeps."""
    n, w, g, m = _muon_list(descs, ws_, gs, ms)
    _check("fp16_muon_step", lib().fp16_muon_step(
        n, descs, w, g, m, float(lr), float(momentum), float(weight_decay), int(bool(nesterov)),
        int(steps), _coef(coef, steps), int(products), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


# ---- dense layers in 8-bit integers -----------------------------------------

INT8_FWD, INT8_BWD, INT8_WEIGHTS = 0, 1, 2


def int8_dense_desc(tokens, inputs, outputs) -> Int8DenseDesc:
    return Int8DenseDesc(int(tokens), int(inputs), int(outputs))


def fp16_int8_row_bytes(n: int) -> int:
    return int(lib().fp16_int8_row_bytes(int(n)))


def int8_operand(rows, n, device="cuda"):
    """Buffers of a quantised operand [rows][n]: its bytes and its scales."""
    import torch
    return (torch.empty((int(rows), fp16_int8_row_bytes(n)), dtype=torch.int8, device=device),
            torch.empty(int(rows), dtype=torch.float32, device=device))


def fp16_int8_quant_rows(rows, cols, x, q, scale, stream=None) -> None:
    _check("fp16_int8_quant_rows", lib().fp16_int8_quant_rows(
        int(rows), int(cols), _ptr_half(x), _ptr_int8(q), _ptr_float(scale), _stream(stream)))


def fp16_int8_quant_workspace_bytes(rows, cols) -> int:
    return int(lib().fp16_int8_quant_workspace_bytes(int(rows), int(cols)))


def fp16_int8_quant_cols(rows, cols, x, q, scale, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_int8_quant_cols", lib().fp16_int8_quant_cols(
        int(rows), int(cols), _ptr_half(x), _ptr_int8(q), _ptr_float(scale), _ptr(ws),
        _wsb(ws, ws_bytes), _stream(stream)))


def fp16_int8_matmul(m, n, k, a, sa, b, sb, bias, y, stream=None) -> None:
    _check("fp16_int8_matmul", lib().fp16_int8_matmul(
        int(m), int(n), int(k), _ptr_int8(a), _ptr_float(sa), _ptr_int8(b), _ptr_float(sb),
        _ptr_half(bias), _ptr_half(y), _stream(stream)))


def fp16_int8_kernel(m, n, k) -> str:
    """The kernel a product runs on (for tests and profiles)."""
    return lib().fp16_int8_kernel(int(m), int(n), int(k)).decode()


def fp16_int8_dense_workspace_bytes(desc: Int8DenseDesc, call=None) -> int:
    """Workspace of one of the layer's calls, or (None) enough for all three."""
    calls = (INT8_FWD, INT8_BWD, INT8_WEIGHTS) if call is None else (int(call),)
    return max(int(lib().fp16_int8_dense_workspace_bytes(ctypes.byref(desc), c)) for c in calls)


def fp16_int8_dense_weights(desc, w, wq, sw, wqt=None, swt=None, ws=None, ws_bytes=None,
                            stream=None) -> None:
    _check("fp16_int8_dense_weights", lib().fp16_int8_dense_weights(
        ctypes.byref(desc), _ptr_half(w), _ptr_int8(wq), _ptr_float(sw), _ptr_int8(wqt),
        _ptr_float(swt), _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_int8_dense_fwd(desc, x, wq, sw, bias, y, ws=None, ws_bytes=None, stream=None) -> None:
    _check("fp16_int8_dense_fwd", lib().fp16_int8_dense_fwd(
        ctypes.byref(desc), _ptr_half(x), _ptr_int8(wq), _ptr_float(sw), _ptr_half(bias),
        _ptr_half(y), _ptr(ws), _wsb(ws, ws_bytes), _stream(stream)))


def fp16_int8_dense_bwd(desc, x, dy, wqt, swt, dx, dw, dbias=None, ws=None, ws_bytes=None,
                        stream=None) -> None:
    _check("fp16_int8_dense_bwd", lib().fp16_int8_dense_bwd(
        ctypes.byref(desc), _ptr_half(x), _ptr_half(dy), _ptr_int8(wqt), _ptr_float(swt),
        _ptr_half(dx), _ptr_half(dw), _ptr_half(dbias), _ptr(ws), _wsb(ws, ws_bytes),
        _stream(stream)))


# ---- dropout from a counter-based generator ---------------------------------

def rng_state(seed, step=0, device="cuda"):
    """The generator's state, [seed, step] (64 bits each, the step advanced by
    fp16_rng_advance or by a program's own arithmetic on element 1)."""
    import torch
    wrap = lambda v: (int(v) + (1 << 63)) % (1 << 64) - (1 << 63)
    return torch.tensor([wrap(seed), wrap(step)], dtype=torch.int64, device=device)


def fp16_rng_advance(rng, steps=1, stream=None) -> None:
    p = _held_long(rng, 2, "rng", _device())
    _check("fp16_rng_advance", lib().fp16_rng_advance(p, int(steps) % (1 << 64), _stream(stream)))


def _fits(what, v, low, high):
    """v, unless a field from low to high would cut it to another number."""
    v = int(v)
    if not low <= v <= high:
        raise ValueError(f"{what} {v}")
    return v


def _int32(**fields):
    return [_fits(k, v, -(1 << 31), (1 << 31) - 1) for k, v in fields.items()]


def fp16_dropout(x, residual, y, p, rng, site=0, n=None, stream=None) -> None:
    """y = dropout of x (+ residual); the gradient is the same call on dy."""
    site = _fits("site", site, 0, 0xFFFFFFFF)
    n = x.numel() if n is None else int(n)
    dev = _device()
    _check("fp16_dropout", lib().fp16_dropout(
        n, _held_half(x, n, "x", dev), _held_half(residual, n, "residual", dev),
        _held_half(y, n, "y", dev), p, _held_long(rng, 2, "rng", dev), site, _stream(stream)))


# ---- dense layers with bias, activation, dropout and residual ----------------

DENSE_FWD, DENSE_BWD = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, None: 0}


def dense_desc(tokens, inputs, outputs, act="none", drop=0.0, site=0) -> DenseDesc:
    """act: a name ("none", "relu", "gelu", "silu") or one of the ACT_ numbers."""
    return DenseDesc(*_int32(tokens=tokens, inputs=inputs, outputs=outputs,
                             act=act if isinstance(act, int) else _ACTS[act]),
                     float(drop), _fits("site", site, 0, 0xFFFFFFFF))


def fp16_dense_workspace_bytes(desc: DenseDesc, call=None) -> int:
    """Workspace of one of the layer's calls, or (None) enough for both."""
    calls = (DENSE_FWD, DENSE_BWD) if call is None else (int(call),)
    return max(int(lib().fp16_dense_workspace_bytes(ctypes.byref(desc), c)) for c in calls)


def fp16_dense_kernel(desc: DenseDesc, product=0) -> str:
    """The kernel that a product runs on (0 forward, 1 dx, 2 dW; for tests and profiles)."""
    return lib().fp16_dense_kernel(ctypes.byref(desc), int(product)).decode()


def fp16_dense_fwd(desc, x, w, bias, residual, y, z=None, rng=None, ws=None, ws_bytes=None,
                   stream=None) -> None:
    t, i, o = desc.tokens, desc.inputs, desc.outputs
    to, dev = t * o, _device()
    work, size = _held_ws(ws, ws_bytes, dev)
    _check("fp16_dense_fwd", lib().fp16_dense_fwd(
        ctypes.byref(desc), _held_half(x, t * i, "x", dev), _held_half(w, o * i, "w", dev),
        _held_half(bias, o, "bias", dev), _held_half(residual, to, "residual", dev),
        _held_long(rng, 2, "rng", dev), _held_half(y, to, "y", dev), _held_half(z, to, "z", dev),
        work, size, _stream(stream)))


def fp16_dense_bwd(desc, x, w, z, dy, dx, dw, dbias=None, rng=None, ws=None, ws_bytes=None,
                   stream=None) -> None:
    t, i, o = desc.tokens, desc.inputs, desc.outputs
    dev = _device()
    work, size = _held_ws(ws, ws_bytes, dev)
    _check("fp16_dense_bwd", lib().fp16_dense_bwd(
        ctypes.byref(desc), _held_half(x, t * i, "x", dev), _held_half(w, o * i, "w", dev),
        _held_half(z, t * o, "z", dev), _held_half(dy, t * o, "dy", dev),
        _held_long(rng, 2, "rng", dev), _held_half(dx, t * i, "dx", dev),
        _held_half(dw, o * i, "dw", dev), _held_half(dbias, o, "dbias", dev),
        work, size, _stream(stream)))


# ---- log probabilities -------------------------------------------------------

LOGPROB_TOP_MAX = 64  # FP16_LOGPROB_TOP_MAX


def logprob_desc(rows, classes, stride=None, scale=1.0, top=0) -> LogprobDesc:
    """stride: elements from row to row (None: classes); scale: one over a temperature."""
    rows, classes, stride, top = _int32(
        rows=rows, classes=classes, stride=classes if stride is None else stride, top=top)
    return LogprobDesc(rows, classes, stride, float(scale), top)


def fp16_logprobs_workspace_bytes(desc: LogprobDesc) -> int:
    return int(lib().fp16_logprobs_workspace_bytes(ctypes.byref(desc)))


def fp16_logprobs(desc, z, tokens, logp, stats, top_id=None, top_logp=None, ws=None,
                  ws_bytes=None, stream=None) -> None:
    """logp, stats [rows][3] (largest logit, log of the sum, entropy) and the desc.top
    most probable classes of each row."""
    n, k, dev = desc.rows, desc.top, _device()
    work, size = _held_ws(ws, ws_bytes, dev)
    _check("fp16_logprobs", lib().fp16_logprobs(
        ctypes.byref(desc), _held_half(z, (n - 1) * desc.stride + desc.classes, "z", dev),
        _held_int(tokens, n, "tokens", dev), _held_float(logp, n, "logp", dev),
        _held_float(stats, 3 * n, "stats", dev), _held_int(top_id, n * k, "top_id", dev),
        _held_float(top_logp, n * k, "top_logp", dev), work, size, _stream(stream)))


def fp16_logprobs_bwd(desc, z, tokens, stats, dlogp, dentropy, dz, stream=None) -> None:
    n, dev = desc.rows, _device()
    size = (n - 1) * desc.stride + desc.classes
    _check("fp16_logprobs_bwd", lib().fp16_logprobs_bwd(
        ctypes.byref(desc), _held_half(z, size, "z", dev), _held_int(tokens, n, "tokens", dev),
        _held_float(stats, 3 * n, "stats", dev), _held_float(dlogp, n, "dlogp", dev),
        _held_float(dentropy, n, "dentropy", dev), _held_half(dz, size, "dz", dev),
        _stream(stream)))


def _wsb(ws, ws_bytes):
    if ws_bytes is not None:
        return int(ws_bytes)
    if ws is None or isinstance(ws, int):
        return 0
    return ws.numel() * ws.element_size()


# ---- conveniences that allocate outputs and workspaces with torch -----------

def workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)
