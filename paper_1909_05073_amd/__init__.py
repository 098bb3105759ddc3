"""Thin Python binding of the PCONV HIP library (argument marshalling and checks only).

Every step of the path - analysis, reorder, compact storage (pconv_pack) and the sparse
convolution (pconv_conv2d) - runs inside libpconv.so; PyTorch appears only as the owner of
device memory and streams.  There is no CPU fallback: if the library is missing or no GPU is
present, calls fail loudly.
"""
from __future__ import annotations

import ctypes as C
import functools
import importlib
import os

import numpy as np

from . import _build

F32, BF16 = 0, 1
NCHW, NHWC = 0, 1
OK, INVALID_ARG, OOM, HIP_ERROR, UNSUPPORTED = 0, -1, -2, -3, -4
MAX_PATTERNS = 16

_DTYPE = {"f32": F32, "bf16": BF16, F32: F32, BF16: BF16}
_LAYOUT = {"nchw": NCHW, "nhwc": NHWC, NCHW: NCHW, NHWC: NHWC}


class PconvError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"pconv status {status}: {message}")
        self.status = status


class pconv_info(C.Structure):
    _fields_ = [("c_out", C.c_int32), ("c_in", C.c_int32), ("num_patterns", C.c_int32),
                ("weight_dtype", C.c_int32), ("kept_kernels", C.c_int64), ("nnz", C.c_int64),
                ("device_bytes", C.c_int64), ("fast_path", C.c_int32), ("reserved", C.c_int32)]


class pconv_plan(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("waves", C.c_int32), ("ks_log2", C.c_int32), ("split_units", C.c_int32),
                ("tail_tiles", C.c_int32), ("flat_shape", C.c_int32), ("lone_patches", C.c_int32), ("lone_cut", C.c_int32)]


class pconv_i8_plan(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("tile_m", C.c_int32), ("tile_n", C.c_int32), ("sets", C.c_int32), ("splits", C.c_int32)]


_lib = None


def library_path() -> str:
    return _build.LIB


def lib():
    """Load libpconv.so (built in-tree by __graft_entry__.build(); built here only if absent)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        _build.build()
    L = C.CDLL(path)
    vp, ip = C.c_void_p, C.c_int
    L.pconv_pack.restype = ip
    L.pconv_pack.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, C.POINTER(vp)]
    L.pconv_project.restype = ip
    L.pconv_project.argtypes = [vp, vp, ip, ip, ip, C.c_int64, vp, vp]
    L.pconv_debug_pack_host.restype = ip
    L.pconv_debug_pack_host.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, C.POINTER(vp)]
    L.pconv_conv2d.restype = ip
    L.pconv_conv2d.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, ip, ip, ip, ip, vp]
    L.pconv_conv2d_static.restype = ip
    L.pconv_conv2d_static.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, ip, ip, ip, ip, vp]
    L.pconv_conv2d_workspace.restype = C.c_int64
    L.pconv_conv2d_workspace.argtypes = [vp, ip, ip, ip, ip, ip, ip]
    L.pconv_conv2d_ws.restype = ip
    L.pconv_conv2d_ws.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, ip, ip, ip, ip, vp, vp, C.c_int64]
    L.pconv_conv2d_or_workspace.restype = C.c_int64
    L.pconv_conv2d_or_workspace.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, ip, ip, ip, ip, vp]
    L.hipThreadExchangeStreamCaptureMode.restype = ip            # (of the HIP runtime, which the library is linked to)
    L.hipThreadExchangeStreamCaptureMode.argtypes = [C.POINTER(ip)]
    L.pconv_conv2d_pool2x2.restype = ip
    L.pconv_conv2d_pool2x2.argtypes = [vp, vp, vp, vp, ip, ip, ip, ip, ip, ip, vp]
    L.pconv_free.restype = None
    L.pconv_free.argtypes = [vp]
    L.pconv_maxpool2x2.restype = ip
    L.pconv_maxpool2x2.argtypes = [vp, vp, ip, ip, ip, ip, ip, ip, vp]
    L.pconv_get_info.restype = ip
    L.pconv_get_info.argtypes = [vp, C.POINTER(pconv_info)]
    L.pconv_debug_export.restype = ip
    L.pconv_debug_export.argtypes = [vp, vp, vp, vp, vp, vp]
    L.pconv_debug_export_blocks.restype = ip
    L.pconv_debug_export_blocks.argtypes = [vp, vp, vp]
    L.pconv_debug_unpack.restype = ip
    L.pconv_debug_unpack.argtypes = [vp, vp]
    L.pconv_set_kernel_policy.restype = ip
    L.pconv_set_kernel_policy.argtypes = [ip]
    L.pconv_debug_set_tiling.restype = ip
    L.pconv_debug_set_tiling.argtypes = [ip, ip, ip]
    L.pconv_debug_set_flat_shape.restype = ip
    L.pconv_debug_set_flat_shape.argtypes = [ip]
    L.pconv_debug_plan.restype = ip
    L.pconv_debug_plan.argtypes = [vp, ip, ip, ip, ip, ip, ip, C.POINTER(pconv_plan)]
    L.pconv_debug_set_spin_limit.restype = ip
    L.pconv_debug_set_spin_limit.argtypes = [ip]
    L.pconv_get_async_error.restype = ip
    L.pconv_get_async_error.argtypes = [vp]
    L.pconv_pool2x2_fusion.restype = ip
    L.pconv_pool2x2_fusion.argtypes = [vp, ip, ip, ip, ip, ip]
    L.pconv_debug_measure_fma_peak.restype = ip
    L.pconv_debug_measure_fma_peak.argtypes = [C.POINTER(C.c_double)]
    i64 = C.c_int64
    L.pconv_quantize_rows.restype = ip
    L.pconv_quantize_rows.argtypes = [vp, i64, ip, i64, i64, vp, i64, vp, vp]
    L.pconv_matmul_i8_workspace.restype = i64
    L.pconv_matmul_i8_workspace.argtypes = [i64, i64, i64, ip]
    L.pconv_matmul_i8.restype = ip
    L.pconv_matmul_i8.argtypes = [vp, i64, vp, vp, i64, vp, vp, vp, i64, ip, i64, i64, i64, ip, vp, i64, vp]
    L.pconv_linear_i8_workspace.restype = i64
    L.pconv_linear_i8_workspace.argtypes = [i64, i64, i64, ip]
    L.pconv_linear_i8.restype = ip
    L.pconv_linear_i8.argtypes = [vp, i64, ip, vp, i64, vp, vp, vp, i64, ip, i64, i64, i64, ip, vp, i64, vp]
    L.pconv_debug_i8_plan.restype = ip
    L.pconv_debug_i8_plan.argtypes = [i64, i64, i64, vp]
    L.pconv_grad_workspace.restype = i64
    L.pconv_grad_workspace.argtypes = [i64]
    L.pconv_grad_norm.restype = ip
    L.pconv_grad_norm.argtypes = [vp, vp, vp, i64, vp, vp, i64, vp]
    L.pconv_clip_grads.restype = ip
    L.pconv_clip_grads.argtypes = [vp, vp, vp, vp, vp, i64, C.c_float, C.c_float, vp, vp, i64, vp]
    L.pconv_last_error.restype = C.c_char_p
    L.pconv_last_error.argtypes = []
    _lib = L
    return L


EXPORTED_SYMBOLS = ["pconv_project", "pconv_pack", "pconv_conv2d", "pconv_conv2d_static", "pconv_conv2d_workspace", "pconv_conv2d_ws", "pconv_conv2d_or_workspace",
                    "pconv_conv2d_pool2x2", "pconv_free", "pconv_maxpool2x2",
                    "pconv_get_info", "pconv_debug_export", "pconv_debug_export_blocks", "pconv_debug_pack_host",
                    "pconv_debug_unpack",
                    "pconv_set_kernel_policy", "pconv_debug_set_tiling", "pconv_debug_set_flat_shape", "pconv_debug_plan", "pconv_debug_set_spin_limit",
                    "pconv_get_async_error", "pconv_pool2x2_fusion", "pconv_debug_measure_fma_peak",
                    "pconv_quantize_rows", "pconv_matmul_i8", "pconv_matmul_i8_workspace", "pconv_linear_i8",
                    "pconv_linear_i8_workspace", "pconv_debug_i8_plan", "pconv_grad_workspace", "pconv_grad_norm", "pconv_clip_grads",
                    "pconv_last_error"]


def _check(rc: int):
    if rc != OK:
        raise PconvError(rc, lib().pconv_last_error().decode())


def _np(a, dt):
    return np.ascontiguousarray(a, dtype=dt)


class Handle:
    """Owns one pconv_handle*; free() or garbage collection releases it."""

    def __init__(self, ptr: int, c_out: int, c_in: int, dtype: int):
        self.ptr, self.c_out, self.c_in, self.dtype = ptr, c_out, c_in, dtype

    def info(self) -> pconv_info:
        out = pconv_info()
        _check(lib().pconv_get_info(self.ptr, C.byref(out)))
        return out

    def free(self):
        if self.ptr:
            lib().pconv_free(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def pconv_pack(w_dense, pattern_id, conn, table, weight_dtype="f32", host_only=False) -> Handle:
    """Host arrays -> packed device handle (see include/pconv.h).

    host_only=True calls pconv_debug_pack_host instead (no GPU needed, no device data)."""
    w = _np(w_dense, np.float32)
    pid = _np(pattern_id, np.uint8)
    cn = _np(conn, np.uint8)
    tb = _np(table, np.uint16)
    if w.ndim != 4 or w.shape[2:] != (3, 3) or pid.shape != w.shape[:2] or cn.shape != w.shape[:2]:
        raise ValueError("expected w [F][C][3][3] and pattern_id/conn [F][C]")
    out = C.c_void_p()
    fn = lib().pconv_debug_pack_host if host_only else lib().pconv_pack
    rc = fn(w.ctypes.data, pid.ctypes.data, cn.ctypes.data, tb.ctypes.data,
            int(tb.size), int(w.shape[0]), int(w.shape[1]), _DTYPE[weight_dtype], C.byref(out))
    _check(rc)
    return Handle(out.value, int(w.shape[0]), int(w.shape[1]), _DTYPE[weight_dtype])


def pconv_project(w_dense, table, keep_kernels: int):
    """Dense weights [F][C][3][3] -> (pattern_id [F][C] uint8, conn [F][C] uint8); see include/pconv.h."""
    w = _np(w_dense, np.float32)
    tb = _np(table, np.uint16)
    if w.ndim != 4 or w.shape[2:] != (3, 3):
        raise ValueError("expected w [F][C][3][3]")
    pid = np.empty(w.shape[:2], np.uint8)
    conn = np.empty(w.shape[:2], np.uint8)
    _check(lib().pconv_project(w.ctypes.data, tb.ctypes.data, int(tb.size), int(w.shape[0]), int(w.shape[1]),
                               int(keep_kernels), pid.ctypes.data, conn.ctypes.data))
    return pid, conn


def pconv_conv2d(handle: Handle, x_ptr: int, y_ptr: int, bias_ptr, n: int, h_in: int, w_in: int,
                 stride: int = 1, pad: int = 1, layout=NCHW, act_dtype=F32, fuse_relu: bool = False,
                 stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_conv2d(handle.ptr, x_ptr, y_ptr, bias_ptr or None, n, h_in, w_in, stride, pad,
                              _LAYOUT[layout], _DTYPE[act_dtype], int(bool(fuse_relu)),
                              stream or None))


def pconv_conv2d_static(handle: Handle, x_ptr: int, y_ptr: int, bias_ptr, n: int, h_in: int, w_in: int,
                        stride: int = 1, pad: int = 1, layout=NCHW, act_dtype=F32, fuse_relu: bool = False,
                        stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_conv2d_static(handle.ptr, x_ptr, y_ptr, bias_ptr or None, n, h_in, w_in, stride, pad,
                                     _LAYOUT[layout], _DTYPE[act_dtype], int(bool(fuse_relu)),
                                     stream or None))


def pconv_conv2d_pool2x2(handle: Handle, x_ptr: int, y_ptr: int, bias_ptr, n: int, h_in: int, w_in: int,
                         layout=NCHW, act_dtype=F32, fuse_relu: bool = False, stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_conv2d_pool2x2(handle.ptr, x_ptr, y_ptr, bias_ptr or None, n, h_in, w_in,
                                      _LAYOUT[layout], _DTYPE[act_dtype], int(bool(fuse_relu)),
                                      stream or None))


def pconv_free(handle: Handle):
    handle.free()


def pconv_maxpool2x2(x_ptr: int, y_ptr: int, n: int, c: int, h: int, w: int, layout=NCHW,
                     dtype=F32, stream: int = 0):
    _check(lib().pconv_maxpool2x2(x_ptr, y_ptr, n, c, h, w, _LAYOUT[layout], _DTYPE[dtype],
                                  stream or None))


def pconv_set_kernel_policy(policy: int):
    """0 automatic, 1 generic gather kernel, 2 register-tiled vector kernel, 3 matrix-core kernel (bf16)."""
    _check(lib().pconv_set_kernel_policy(int(policy)))


def pconv_debug_set_tiling(waves: int = 0, ks_log2: int = -1, split_units: int = -1):
    _check(lib().pconv_debug_set_tiling(int(waves), int(ks_log2), int(split_units)))


def pconv_debug_set_flat_shape(index: int = -1):
    _check(lib().pconv_debug_set_flat_shape(int(index)))


def pconv_debug_plan(handle: Handle, n: int, h_in: int, w_in: int, stride: int = 1, layout=NCHW,
                     fuse_pool: bool = False) -> pconv_plan:
    out = pconv_plan()
    _check(lib().pconv_debug_plan(handle.ptr, n, h_in, w_in, stride, _LAYOUT[layout], int(bool(fuse_pool)), C.byref(out)))
    return out


def pconv_pool2x2_fusion(handle: Handle, n: int, h_in: int, w_in: int, layout=NCHW, act_dtype=F32) -> int:
    """0 = the fused call is not supported, 1 = supported but not recommended, 2 = recommended."""
    rc = lib().pconv_pool2x2_fusion(handle.ptr, n, h_in, w_in, _LAYOUT[layout], _DTYPE[act_dtype])
    if rc < 0:
        _check(rc)
    return rc


def pconv_debug_measure_fma_peak() -> float:
    out = C.c_double()
    _check(lib().pconv_debug_measure_fma_peak(C.byref(out)))
    return out.value


def pconv_debug_set_spin_limit(limit: int = 0):
    _check(lib().pconv_debug_set_spin_limit(int(limit)))


def pconv_get_async_error(handle: Handle):
    """Raises PconvError(HIP_ERROR) once if a kernel on this handle gave up a bounded wait."""
    _check(lib().pconv_get_async_error(handle.ptr))


def pconv_debug_export_blocks(handle: Handle):
    """(slot_filter [B][4] int32, records [B][J] uint32): see include/pconv.h."""
    info = handle.info()
    b, j = -(-info.c_out // 4), -(-info.c_in // 8)
    slot_filter = np.empty((b, 4), np.int32); records = np.empty((b, j), np.uint32)
    _check(lib().pconv_debug_export_blocks(handle.ptr, slot_filter.ctypes.data, records.ctypes.data))
    return slot_filter, records


def pconv_debug_export(handle: Handle) -> dict:
    info = handle.info()
    f, p = info.c_out, info.num_patterns
    perm = np.empty(f, np.uint16); row_ptr = np.empty(f + 1, np.uint32)
    pat_cnt = np.empty((f, p), np.uint16); cin = np.empty(info.kept_kernels, np.uint16)
    vals = np.empty(info.nnz, np.float32 if info.weight_dtype == F32 else np.uint16)
    _check(lib().pconv_debug_export(handle.ptr, perm.ctypes.data, row_ptr.ctypes.data,
                                    pat_cnt.ctypes.data, cin.ctypes.data, vals.ctypes.data))
    return dict(perm=perm, row_ptr=row_ptr, pat_cnt=pat_cnt, cin=cin, vals=vals)


def pconv_debug_unpack(handle: Handle) -> np.ndarray:
    w = np.empty((handle.c_out, handle.c_in, 3, 3), np.float32)
    _check(lib().pconv_debug_unpack(handle.ptr, w.ctypes.data))
    return w


# ---- torch conveniences (device memory + streams only) ---------------------------------

_raw_stream = None


def _stream(index: int):
    """torch's current stream on device `index`, as the C entry points take it."""
    # (a stream object costs 1.9 us, more than everything else around a call but the launch)
    global _raw_stream
    if _raw_stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream = raw or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(index) or None


def conv2d(handle: Handle, x, bias=None, stride: int = 1, relu: bool = False, layout="nchw",
           out=None):
    """x: CUDA tensor (NCHW or NHWC contiguous). Returns y on the same device/stream."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor")
    lay = _LAYOUT[layout]
    if lay == NCHW:
        n, c, h, w = x.shape
    else:
        n, h, w, c = x.shape
    if c != handle.c_in:
        raise ValueError("channel count does not match the handle")
    dtype = handle.dtype
    if x.dtype != (torch.float32 if dtype == F32 else torch.bfloat16):
        raise ValueError("activation dtype does not match the handle")
    if out is None:
        ho, wo = (h - 1) // stride + 1, (w - 1) // stride + 1
        shape = (n, handle.c_out, ho, wo) if lay == NCHW else (n, ho, wo, handle.c_out)
        out = torch.empty(shape, dtype=x.dtype, device=x.device)
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_cuda):
        raise ValueError("bias must be a float32 CUDA tensor")
    if lay == NHWC and dtype == F32:
        return _conv2d_ws(handle, x, bias, stride, relu, out, n, h, w)
    rc = (_lib or lib()).pconv_conv2d(handle.ptr, x.data_ptr(), out.data_ptr(), (bias.data_ptr() or None) if bias is not None else None,
                                      n, h, w, stride, 1, lay, dtype, 1 if relu else 0, _stream(x.get_device()))
    if rc != OK:
        _check(rc)
    return out


_CAPTURE_MODE_RELAXED = 2                            # hipStreamCaptureModeRelaxed


def _graph_pool_serves(device) -> bool:
    """While the current stream is being captured: whether torch's allocator knows and serves it out of the graph's own pool.

    A graph that is captured otherwise keeps the address of a tensor that is gone when the call returns.  Such a
    capture in HIP's global or thread-local mode is made invalid by the queries of events that the allocator may have
    outstanding, so it is asked in the relaxed mode."""
    import torch
    mode = C.c_int(_CAPTURE_MODE_RELAXED)
    exchange = (_lib or lib()).hipThreadExchangeStreamCaptureMode
    if exchange(C.byref(mode)) != 0:
        return False
    try:
        at = torch.empty(1, dtype=torch.uint8, device=device).data_ptr()
        return any(s["address"] <= at < s["address"] + s["total_size"] and tuple(s["segment_pool_id"]) != (0, 0)
                   for s in torch.cuda.memory_snapshot())
    except (RuntimeError, KeyError):
        return False
    finally:
        exchange(C.byref(mode))


def _conv2d_ws(handle: Handle, x, bias, stride, relu, out, n, h, w):
    """conv2d of fp32 tensors with channels last: lends the call work space out of torch's pool, if there is any.

    Up to the size of x and out together.  On a card with less to spare torch first gives its cached blocks back, which
    waits for the device, and the call then runs without; pconv_conv2d takes none in the first place."""
    L = _lib or lib()
    ptr, c = handle.ptr, handle.c_in
    call = (ptr, x.data_ptr(), out.data_ptr(), (bias.data_ptr() or None) if bias is not None else None,
            n, h, w, stride, 1, NHWC, F32, 1 if relu else 0, _stream(x.get_device()))
    if c > 16 or (c > 4 and c % 4):                  # (mostly some)
        size = L.pconv_conv2d_workspace(ptr, n, h, w, stride, NHWC, F32)
    else:                                            # (mostly none: question and call are one; 4.8 us on the host for 5.6)
        size = L.pconv_conv2d_or_workspace(*call)
        if size <= 0:
            if size != OK:
                _check(size)
            return out
    import torch
    work = None
    if size > 0 and torch.cuda.is_current_stream_capturing() and not _graph_pool_serves(x.device):
        size = 0
    if size > 0:
        try:
            work = torch.empty(size, dtype=torch.uint8, device=x.device)
        except torch.cuda.OutOfMemoryError:
            size = 0
    rc = L.pconv_conv2d_ws(*call, work.data_ptr() if work is not None else None, size)
    if rc != OK:
        _check(rc)
    return out


def conv2d_pool2x2(handle: Handle, x, bias=None, relu: bool = False, out=None):
    """x: contiguous fp32 NCHW CUDA tensor.  Returns maxpool2x2(conv2d(x)) without the intermediate."""
    import torch
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor")
    n, c, h, w = x.shape
    if c != handle.c_in:
        raise ValueError("channel count does not match the handle")
    if x.dtype != (torch.float32 if handle.dtype == F32 else torch.bfloat16):
        raise ValueError("activation dtype does not match the handle")
    y = out if out is not None else torch.empty((n, handle.c_out, h // 2, w // 2), dtype=x.dtype, device=x.device)
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_cuda):
        raise ValueError("bias must be a float32 CUDA tensor")
    pconv_conv2d_pool2x2(handle, x.data_ptr(), y.data_ptr(), bias.data_ptr() if bias is not None else 0,
                         n, h, w, NCHW, handle.dtype, relu, _stream(x.get_device()))
    return y


def maxpool2x2(x, layout="nchw"):
    import torch
    if not x.is_cuda:                                # (its address would be a host address to the kernel)
        raise ValueError("x must be a CUDA tensor")
    lay = _LAYOUT[layout]
    if lay == NCHW:
        n, c, h, w = x.shape
        shape = (n, c, h // 2, w // 2)
    else:
        n, h, w, c = x.shape
        shape = (n, h // 2, w // 2, c)
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    dt = F32 if x.dtype == torch.float32 else BF16
    pconv_maxpool2x2(x.data_ptr(), y.data_ptr(), n, c, h, w, lay, dt,
                     _stream(x.get_device()))
    return y


# ---- layers in 8-bit integers ------------------------------------------------------------
#
# They serve networks that are trained: nothing is recorded for autograd, and results ask for no gradient whatever the inputs do.

_types = {}                                          # torch's types to the library's; filled by the first call


def _type_of(t, what):
    code = _types.get(t.dtype)
    if code is None:
        import torch
        _types.update({torch.float32: F32, torch.bfloat16: BF16})
        code = _types.get(t.dtype)
        if code is None:
            raise ValueError(f"{what} must be float32 or bfloat16")
    return code


_current_device = None


def _device_index(*tensors) -> int:
    """The one device that the tensors (or None) are on, which has to be torch's current one."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    at = None
    for t in tensors:
        if t is None:
            continue
        i = t.get_device()                               # (-1 on the host)
        if i < 0:
            raise ValueError("all tensors must be CUDA tensors")
        if at is None:
            at = i
        elif i != at:
            raise ValueError("all tensors must be on one device")
    if at is None:
        return -1
    if at != _current_device():
        raise ValueError("the tensors' device must be the current one")
    return at


def _rows(t, what):
    """(rows, columns, elements from row to row) of a tensor [..., columns] whose rows can be walked with one stride."""
    shape = t.shape
    if len(shape) != 2:
        if not shape:
            raise ValueError(f"{what} must have at least one dimension")
        k = shape[-1]
        if t.is_contiguous():
            return (t.numel() // k if k else _prod(shape[:-1])), k, k
        try:
            t = t.view(-1, k)
        except RuntimeError:
            raise ValueError(f"the rows of {what} must lie one stride apart") from None
        shape = t.shape
    m, k = shape
    step, one = t.stride()
    if one != 1 and k > 1:
        raise ValueError(f"{what} must be contiguous along its last dimension")
    if step < k:
        if m > 1:
            raise ValueError(f"the rows of {what} must not overlap")
        step = k
    return m, k, step


def _prod(sizes) -> int:
    n = 1
    for s in sizes:
        n *= s
    return n


def _scratch(size: int, like):
    """Work space out of torch's pool for a call on the current stream."""
    import torch
    if torch.cuda.is_current_stream_capturing() and not _graph_pool_serves(like.device):
        raise RuntimeError("the stream is being captured by others than torch: call the pconv_... function with work space of your own")
    return torch.empty_strided((size,), (1,), dtype=torch.uint8, device=like.device)


def _per_channel(t, n, what):
    import torch
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be {n} contiguous float32 numbers")
    return t.data_ptr() or None


def _empty(lead, m, n, dtype, like):
    """A new tensor [..., n] of m rows.  (For [m, n] by sizes and steps: 0.5 us less than by its shape.)"""
    import torch
    if len(lead) == 1:
        return torch.empty_strided((m, n), (n or 1, 1), dtype=dtype, device=like.device)
    return like.new_empty(lead + (n,), dtype=dtype)


def _output(out, lead, m, n, dtype, like):
    """(tensor, elements from row to row) for a result [..., n] of m rows."""
    if out is None:
        return _empty(lead, m, n, dtype, like), n
    shape = lead + (n,)
    if out.dtype != dtype or out.shape != shape:
        raise ValueError(f"out must be {dtype} of shape {tuple(shape)}")
    return out, _rows(out, "out")[2]


def _share(a, b) -> bool:
    """Whether two runs of rows, (address, rows, bytes of a row, bytes from row to row), have a byte in common."""
    (at, rows, size, step), (to, others, length, apart) = a, b
    if not (rows and size and others and length):
        return False
    if at >= to + (others - 1) * apart + length or to >= at + (rows - 1) * step + size:
        return False
    if rows == 1:
        step = apart
    elif others == 1:
        apart = step
    # Of the second run's rows the first that ends behind the start of a row of the first run must begin behind its end.
    # With equal distances only how many rows further it is counts, so that one row stands for all.
    if step == apart:
        j = max((at - to - length) // apart + 1, 1 - rows)
        return j < others and to + j * apart < at + size
    starts = at + step * np.arange(rows, dtype=np.int64)
    j = np.maximum((starts - to - length) // apart + 1, 0)
    return bool(((j < others) & (to + j * apart < starts + size)).any())


_tensors_module = None


def _tensor_list_calls():
    """csrc/pconv_tensors.cpp, what is asked of many tensors at once (built as lib() is)."""
    global _tensors_module
    if _tensors_module is None:
        import torch                                     # noqa: F401  (its libraries, which the module needs)
        if not os.path.exists(_build.TENSORS):
            _build.build_tensors()
        _tensors_module = importlib.import_module("._tensors", __name__)
    return _tensors_module


def _refuse_overlap(out, *inputs):
    """out and each of the inputs: (tensor or None, rows, columns, elements from row to row)."""
    run = lambda t, rows, columns, step: (t.data_ptr(), rows, columns * t.element_size(), step * t.element_size())
    to = run(*out)
    for i in inputs:
        if i[0] is not None and _share(to, run(*i)):
            raise ValueError("out must not overlap an input")


def pconv_quantize_rows(x_ptr: int, x_stride: int, x_dtype, rows: int, cols: int, q_ptr: int, q_stride: int,
                        scale_ptr: int, stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_quantize_rows(x_ptr or None, x_stride, _DTYPE[x_dtype], rows, cols, q_ptr or None, q_stride,
                                     scale_ptr or None, stream or None))


def pconv_matmul_i8_workspace(m: int, n: int, k: int, rows_at_16: bool = False) -> int:
    return lib().pconv_matmul_i8_workspace(m, n, k, int(bool(rows_at_16)))


def pconv_matmul_i8(a_ptr: int, a_stride: int, a_scale: int, b_ptr: int, b_stride: int, b_scale: int, bias_ptr, y_ptr: int,
                    y_stride: int, y_dtype, m: int, n: int, k: int, fuse_relu: bool = False, work: int = 0,
                    work_bytes: int = 0, stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_matmul_i8(a_ptr or None, a_stride, a_scale or None, b_ptr or None, b_stride, b_scale or None,
                                 bias_ptr or None, y_ptr or None, y_stride, _DTYPE[y_dtype], m, n, k, int(bool(fuse_relu)),
                                 work or None, work_bytes, stream or None))


def pconv_linear_i8_workspace(m: int, n: int, k: int, rows_at_16: bool = False) -> int:
    return lib().pconv_linear_i8_workspace(m, n, k, int(bool(rows_at_16)))


def pconv_linear_i8(x_ptr: int, x_stride: int, x_dtype, w_ptr: int, w_stride: int, w_scale: int, bias_ptr, y_ptr: int,
                    y_stride: int, y_dtype, m: int, n: int, k: int, fuse_relu: bool = False, work: int = 0,
                    work_bytes: int = 0, stream: int = 0):
    """Raw-pointer call, one to one with the C entry point."""
    _check(lib().pconv_linear_i8(x_ptr or None, x_stride, _DTYPE[x_dtype], w_ptr or None, w_stride, w_scale or None,
                                 bias_ptr or None, y_ptr or None, y_stride, _DTYPE[y_dtype], m, n, k, int(bool(fuse_relu)),
                                 work or None, work_bytes, stream or None))


def pconv_debug_i8_plan(m: int, n: int, k: int) -> pconv_i8_plan:
    out = pconv_i8_plan()
    _check(lib().pconv_debug_i8_plan(m, n, k, C.byref(out)))
    return out


# (remembered by sizes: a call of the library costs 0.7 us)
_linear_i8_workspace = functools.lru_cache(maxsize=4096)(pconv_linear_i8_workspace)
_matmul_i8_workspace = functools.lru_cache(maxsize=4096)(pconv_matmul_i8_workspace)


def _at_16(ptr: int, step: int) -> bool:
    return (ptr | step) & 15 == 0 and step <= 1 << 23


def quantize_rows(x):
    """x: CUDA tensor [..., k], fp32 or bf16.  Returns (q [..., k] int8, scale [...] fp32): x is about q * scale[..., None].

    The rows of q lie a multiple of 16 bytes apart, as matmul_i8 and linear_i8 read them fastest.  Nothing is recorded for autograd."""
    import torch
    dtype = _type_of(x, "x")
    index = _device_index(x)
    m, k, step = _rows(x, "x")
    lead = x.shape[:-1]
    wide = (k + 15) // 16 * 16
    q = _empty(lead, m, wide, torch.int8, x)
    scale = torch.empty_strided((m,), (1,), dtype=torch.float32, device=x.device) if len(lead) == 1 else x.new_empty(lead, dtype=torch.float32)
    rc = (_lib or lib()).pconv_quantize_rows(x.data_ptr() or None, step, dtype, m, k, q.data_ptr() or None, wide,
                                             scale.data_ptr() or None, _stream(index))
    if rc != OK:
        _check(rc)
    return (q if wide == k else q[..., :k]), scale


def matmul_i8(a, a_scale, b, b_scale, bias=None, relu: bool = False, out_dtype=None, out=None):
    """a [..., k], b [n, k]: int8 CUDA tensors.  Returns act((a @ b.T) * a_scale[..., None] * b_scale + bias) [..., n].

    a_scale [...], b_scale [n], bias [n]: fp32.  out_dtype: torch.float32 (unless `out` says otherwise) or torch.bfloat16.
    out: where the result goes; it must not overlap an input (its rows may lie between those of one).  Nothing is recorded for
    autograd."""
    import torch
    if a.dtype != torch.int8 or b.dtype != torch.int8 or b.dim() != 2:
        raise ValueError("a [..., k] and b [n, k] must be int8")
    index = _device_index(a, a_scale, b, b_scale, bias, out)
    m, k, a_step = _rows(a, "a")
    n, kb, b_step = _rows(b, "b")
    if k != kb:
        raise ValueError("a and b must have rows of one length")
    if out_dtype is None:
        out_dtype = out.dtype if out is not None else torch.float32
    y, y_step = _output(out, a.shape[:-1], m, n, out_dtype, a)
    y_type = _type_of(y, "out")
    sa, sb = _per_channel(a_scale, m, "a_scale"), _per_channel(b_scale, n, "b_scale")
    bp = _per_channel(bias, n, "bias") if bias is not None else None
    if out is not None and not _tensor_list_calls().apart(y, a, b, a_scale, b_scale, bias):
        _refuse_overlap((y, m, n, y_step), (a, m, k, a_step), (b, n, k, b_step), (a_scale, 1, m, m), (b_scale, 1, n, n), (bias, 1, n, n))
    a_ptr, b_ptr = a.data_ptr(), b.data_ptr()
    size = _matmul_i8_workspace(m, n, k, _at_16(a_ptr, a_step) and _at_16(b_ptr, b_step))
    work = _scratch(size, a) if size else None
    rc = (_lib or lib()).pconv_matmul_i8(a_ptr or None, a_step, sa, b_ptr or None, b_step, sb, bp, y.data_ptr() or None, y_step,
                                         y_type, m, n, k, 1 if relu else 0, work.data_ptr() if size else None, size,
                                         _stream(index))
    if rc != OK:
        _check(rc)
    if out is not None:
        _tensor_list_calls().changed([y])
    return y


def linear_i8(x, w, w_scale, bias=None, relu: bool = False, out_dtype=None, out=None):
    """x [..., k]: CUDA tensor, fp32 or bf16; w [n, k] int8 and w_scale [n] as quantize_rows gives them for the weights.

    Returns matmul_i8(*quantize_rows(x), w, w_scale, bias, relu) [..., n], of x's type unless `out_dtype` or `out` says
    otherwise.  out: as there.  Nothing is recorded for autograd."""
    import torch
    x_type = _type_of(x, "x")
    if w.dtype != torch.int8 or w.dim() != 2:
        raise ValueError("w [n, k] must be int8")
    index = _device_index(x, w, w_scale, bias, out)
    m, k, x_step = _rows(x, "x")
    n, kw, w_step = _rows(w, "w")
    if k != kw:
        raise ValueError("x and w must have rows of one length")
    if out is None and out_dtype is None:
        y, y_step, y_type = x.new_empty(m, n) if x.dim() == 2 else x.new_empty(x.shape[:-1] + (n,)), n, x_type
    else:
        y, y_step = _output(out, x.shape[:-1], m, n, out_dtype or out.dtype, x)
        y_type = _type_of(y, "out")
    sw = _per_channel(w_scale, n, "w_scale")
    bp = _per_channel(bias, n, "bias") if bias is not None else None
    if out is not None and not _tensor_list_calls().apart(y, x, w, w_scale, bias):
        _refuse_overlap((y, m, n, y_step), (x, m, k, x_step), (w, n, k, w_step), (w_scale, 1, n, n), (bias, 1, n, n))
    w_ptr = w.data_ptr()
    size = _linear_i8_workspace(m, n, k, _at_16(w_ptr, w_step))
    work = _scratch(size, x) if size else None
    rc = (_lib or lib()).pconv_linear_i8(x.data_ptr() or None, x_step, x_type, w_ptr or None, w_step, sw, bp,
                                         y.data_ptr() or None, y_step, y_type, m, n, k, 1 if relu else 0,
                                         work.data_ptr() if size else None, size, _stream(index))
    if rc != OK:
        _check(rc)
    if out is not None:
        _tensor_list_calls().changed([y])
    return y


# ---- gradients of a training step ----------------------------------------------------------

def pconv_grad_workspace(num: int) -> int:
    return lib().pconv_grad_workspace(num)


def pconv_grad_norm(grads, counts, dtypes, num: int, norm_ptr: int, work: int, work_bytes: int, stream: int = 0):
    """Raw call, one to one with the C entry point; the first three are ctypes arrays."""
    _check(lib().pconv_grad_norm(grads, counts, dtypes, num, norm_ptr or None, work or None, work_bytes, stream or None))


def pconv_clip_grads(grads, outs, counts, dtypes, out_dtypes, num: int, max_norm: float, eps: float, norm_ptr: int, work: int,
                     work_bytes: int, stream: int = 0):
    """Raw call, one to one with the C entry point; the first five are ctypes arrays."""
    _check(lib().pconv_clip_grads(grads, outs, counts, dtypes, out_dtypes, num, max_norm, eps, norm_ptr or None, work or None,
                                  work_bytes, stream or None))


def _dense(t) -> bool:
    """Whether the tensor's elements fill one run of memory, each place once, in whatever order of dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for step, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if step != want:
            return False
        want *= size
    return True


class GradList:
    """The gradients of a network's tensors, to be measured and limited together.

    grads: CUDA tensors on one device, fp32 or bf16, each dense (contiguous in some order of its dimensions).  out: where
    the limited gradients go, a tensor of the same shape and strides, fp32 or bf16, for each; without it they are
    changed in place.

    The list keeps the tensors.  Every call looks whether one of them was given other memory, sizes or another type (`data`,
    `set_`, `resize_`), and follows it there.  Gradients that are replaced by other tensors, as
    zero_grad(set_to_none=True), torch's default, does, need a new list: this one goes on limiting the old ones.  (To make
    one takes some 1 us a tensor.)"""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        self._writes = True
        self._lay_out()

    @classmethod
    def _read_only(cls, grads):
        """A list whose norm alone is asked for: its tensors may overlap."""
        made = cls.__new__(cls)
        made.grads = made.out = list(grads)
        made._writes = False
        made._lay_out()
        return made

    def _lay_out(self):
        """Checks the tensors, and writes down where they lie as the library takes it."""
        self._at = None                                  # (until all of them are found right)
        grads, outs = self.grads, self.out
        if len(outs) != len(grads):
            raise ValueError("out must hold a tensor for each gradient")
        self._index = _device_index(*grads, *(outs if outs is not grads else ()))
        for g, o in zip(grads, outs):
            if not _dense(g):
                raise ValueError("a gradient must be dense")
            if o is not g and (o.shape != g.shape or (o.stride() != g.stride() and o.numel() > 1 and
                                                      not (o.is_contiguous() and g.is_contiguous()))):
                raise ValueError("an output must have the shape and the strides of its gradient")
        num = self._num = len(grads)
        types = [_type_of(g, "gradients") for g in grads]
        out_types = [_type_of(o, "outputs") for o in outs]
        self._counts = (C.c_int64 * num)(*(g.numel() for g in grads))
        self._in = (C.c_void_p * num)(*(g.data_ptr() for g in grads))
        self._to = (C.c_void_p * num)(*(o.data_ptr() for o in outs))
        self._types, self._out_types = (C.c_int32 * num)(*types), (C.c_int32 * num)(*out_types)
        if self._writes:
            self._refuse_overlaps(types, out_types)
        self._size = lib().pconv_grad_workspace(num)
        self._tensors = _tensor_list_calls()
        self._at = self._tensors.places(grads, outs)

    def _refuse_overlaps(self, types, out_types):
        """No output may lie over another one, or over a gradient that is not its own."""
        runs = []
        for g, o, n, tg, to in zip(self._in, self._to, self._counts, types, out_types):
            if n:
                runs.append((o, o + n * (2 if to == BF16 else 4), True))
                if (g, tg) != (o, to):
                    runs.append((g, g + n * (2 if tg == BF16 else 4), False))
        any_end = out_end = 0
        for start, end, written in sorted(runs):
            if start < (any_end if written else out_end):
                raise ValueError("outputs overlap each other or other gradients")
            any_end = max(any_end, end)
            if written:
                out_end = max(out_end, end)

    def _begin(self):
        import torch
        if self._tensors.places(self.grads, self.out) != self._at:
            self._lay_out()
        if self._num == 0:
            raise ValueError("the list is empty")
        like = self.grads[0]
        if self._index != _current_device():
            raise ValueError("the tensors' device must be the current one")
        work = _scratch(self._size, like)
        return torch.empty_strided((), (), dtype=torch.float32, device=like.device), work

    def norm(self):
        """The 2-norm of all gradients together, a tensor of one fp32 number on their device."""
        norm, work = self._begin()
        rc = (_lib or lib()).pconv_grad_norm(self._in, self._counts, self._types, self._num, norm.data_ptr(), work.data_ptr(),
                                             self._size, _stream(self._index))
        if rc != OK:
            _check(rc)
        return norm

    def clip(self, max_norm: float, eps: float = 1e-6):
        """Multiplies all gradients by min(1, max_norm / (norm + eps)).  Returns the norm, as norm() does."""
        norm, work = self._begin()
        rc = (_lib or lib()).pconv_clip_grads(self._in, self._to, self._counts, self._types, self._out_types, self._num,
                                              max_norm, eps, norm.data_ptr(), work.data_ptr(), self._size,
                                              _stream(self._index))
        if rc != OK:
            _check(rc)
        self._tensors.changed(self.out)
        return norm


def grad_norm(grads):
    """The 2-norm of all gradients together; see GradList.  Nothing is written, and the tensors may overlap."""
    return GradList._read_only(grads).norm()


def clip_grad_norm(grads, max_norm: float, eps: float = 1e-6, out=None):
    """Limits the norm of all gradients together, in place unless `out` says otherwise; see GradList.  Returns the norm."""
    return GradList(grads, out).clip(max_norm, eps)
