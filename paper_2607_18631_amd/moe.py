"""Thin ctypes binding of libmoe_mi355x.so (include/moe.h), same names as the C ABI.

Argument marshalling only: every step of the layer runs in the library's HIP kernels.
Tensors are torch device tensors (torch provides device memory and streams); each call
passes their data pointers and the current torch stream.  If the library is not built,
``lib()`` raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from .workloads import MoEShape

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmoe_mi355x.so")

MOE_OK, MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP = range(5)
(MOE_WS_ROUTE, MOE_WS_PERMUTE, MOE_WS_FFN, MOE_WS_LAYER, MOE_WS_FFN_BWD, MOE_WS_LAYER_BWD, MOE_WS_MX_FFN,
 MOE_WS_DECODE) = range(8)
MOE_MX_E2M1, MOE_MX_E4M3 = range(2)
MOE_DECODE_MAX_TOKENS = 64
MOE_FUSION_SET, MOE_FUSE_GATHER, MOE_FUSE_COMBINE = 0x10, 0x1, 0x2
(MOE_REGION_TOPK_IDX, MOE_REGION_TOPK_W, MOE_REGION_COUNTS, MOE_REGION_OFFSETS, MOE_REGION_ROW_TOKEN,
 MOE_REGION_SLOT_ROW, MOE_REGION_X_PERM, MOE_REGION_Y_PERM, MOE_REGION_SHARED_Y) = range(9)

EXPORTS = ["moe_abi_version", "moe_status_string", "moe_last_error", "moe_workspace_size",
           "moe_workspace_offset", "moe_route", "moe_permute", "moe_grouped_ffn", "moe_combine",
           "moe_layer_forward", "moe_layer_forward_traced", "moe_grouped_ffn_backward", "moe_layer_backward",
           "moe_permute_noalloc", "moe_mx_quantize", "moe_mx_dequantize", "moe_mx_grouped_ffn", "moe_add_rmsnorm",
           "moe_add_rmsnorm_backward", "moe_add_rmsnorm_workspace_size", "moe_layer_decode"]
MOE_STEP_NAMES = ["router_gemm", "gate", "histogram", "permute", "ffn_up", "ffn_down", "shared_up",
                  "shared_down", "combine"]


class MoEShapeC(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d", ctypes.c_int32), ("E", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("e_begin", ctypes.c_int32), ("E_local", ctypes.c_int32),
                ("F", ctypes.c_int32), ("F_shared", ctypes.c_int32), ("gate", ctypes.c_int32),
                ("n_group", ctypes.c_int32), ("topk_group", ctypes.c_int32),
                ("renormalize", ctypes.c_int32), ("routed_scale", ctypes.c_float),
                ("expert_capacity", ctypes.c_int32), ("fusion", ctypes.c_int32)]


class MoEError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"status {status}: {message}")
        self.status = status


_lib = None
_vp = ctypes.c_void_p
# torch's names that the calls below take, from lib() on (importing this module does not import torch)
_bf16 = _f32 = _i32 = _u8 = _raw_stream = _current_device = None


def lib():
    """Load the built library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2607_18631_amd.build)")
        # torch ships its own HIP runtime under the same soname (libamdhip64.so.7) as the system
        # one the library is linked against.  Loading torch first makes the library bind to that
        # runtime; loaded the other way round, the process holds two runtimes and the library's
        # kernels are not found for torch's device memory ("invalid device function").
        import torch
        global _bf16, _f32, _i32, _u8, _raw_stream, _current_device
        _bf16, _f32, _i32, _u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
        _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
        L = ctypes.CDLL(LIB_PATH)
        sp = ctypes.POINTER(MoEShapeC)
        L.moe_abi_version.restype = ctypes.c_int
        L.moe_status_string.restype = ctypes.c_char_p
        L.moe_status_string.argtypes = [ctypes.c_int]
        L.moe_last_error.restype = ctypes.c_char_p
        L.moe_workspace_size.restype = ctypes.c_size_t
        L.moe_workspace_size.argtypes = [sp, ctypes.c_int]
        L.moe_workspace_offset.restype = ctypes.c_size_t
        L.moe_workspace_offset.argtypes = [sp, ctypes.c_int]
        L.moe_route.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.moe_permute.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.moe_grouped_ffn.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.moe_permute_noalloc.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
        L.moe_combine.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp]
        L.moe_grouped_ffn_backward.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t,
                                               _vp]
        L.moe_layer_backward.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t,
                                         _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.moe_layer_forward.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.moe_layer_forward_traced.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t,
                                               ctypes.POINTER(_vp), _vp]
        sz, i32, i64, f32 = ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        L.moe_mx_quantize.argtypes = [i64, i32, i32, _vp, _vp, _vp, _vp]
        L.moe_mx_dequantize.argtypes = [i64, i32, i32, _vp, _vp, _vp, _vp]
        L.moe_mx_grouped_ffn.argtypes = [sp, i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, sz, _vp]
        L.moe_add_rmsnorm.argtypes = [i64, i32, f32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
        L.moe_add_rmsnorm_backward.argtypes = [i64, i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, sz, _vp]
        L.moe_add_rmsnorm_workspace_size.argtypes = [i64, i32]
        L.moe_add_rmsnorm_workspace_size.restype = sz
        L.moe_layer_decode.argtypes = [sp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, sz, _vp]
        for f in ("moe_route", "moe_permute", "moe_grouped_ffn", "moe_combine", "moe_layer_forward",
                  "moe_layer_forward_traced", "moe_grouped_ffn_backward", "moe_layer_backward", "moe_mx_quantize",
                  "moe_mx_dequantize", "moe_mx_grouped_ffn", "moe_add_rmsnorm", "moe_add_rmsnorm_backward",
                  "moe_layer_decode"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def shape_c(sh: MoEShape) -> MoEShapeC:
    return MoEShapeC(sh.T, sh.d, sh.E, sh.top_k, sh.e_begin, sh.E_local, sh.F, sh.F_shared, sh.gate,
                     sh.n_group, sh.topk_group, sh.renormalize, sh.routed_scale, sh.expert_capacity,
                     sh.fusion)


def last_error() -> str:
    return lib().moe_last_error().decode()


def _check(status: int):
    if status != MOE_OK:
        raise MoEError(status, last_error())


def _p(t):
    """Data pointer of a tensor (or None)."""
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream)
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def workspace_size(sh: MoEShape, kind: int) -> int:
    n = lib().moe_workspace_size(ctypes.byref(shape_c(sh)), kind)
    if n == 0:
        raise MoEError(MOE_ERR_INVALID_ARG, last_error())
    return n


def workspace_offset(sh: MoEShape, region: int) -> int:
    n = lib().moe_workspace_offset(ctypes.byref(shape_c(sh)), region)
    if n == ctypes.c_size_t(-1).value:
        raise MoEError(MOE_ERR_INVALID_ARG, last_error())
    return n


def alloc_workspace(sh: MoEShape, kind: int, device="cuda"):
    import torch
    return torch.empty(workspace_size(sh, kind), dtype=torch.uint8, device=device)


def moe_route(sh, x, w_router, bias, topk_idx, topk_w, keys_out=None, ws=None, stream=None):
    _check(lib().moe_route(ctypes.byref(shape_c(sh)), _p(x), _p(w_router), _p(bias), _p(topk_idx), _p(topk_w),
                           _p(keys_out), _p(ws), 0 if ws is None else ws.numel(), _stream(stream)))


def moe_permute(sh, topk_idx, x, counts, offsets, row_token, slot_row, x_perm, ws=None, stream=None):
    _check(lib().moe_permute(ctypes.byref(shape_c(sh)), _p(topk_idx), _p(x), _p(counts), _p(offsets),
                             _p(row_token), _p(slot_row), _p(x_perm), _p(ws), 0 if ws is None else ws.numel(),
                             _stream(stream)))


def moe_permute_noalloc(sh, topk_idx, x, counts, offsets, row_token, slot_row, x_perm, stream=None):
    _check(lib().moe_permute_noalloc(ctypes.byref(shape_c(sh)), _p(topk_idx), _p(x), _p(counts), _p(offsets),
                                     _p(row_token), _p(slot_row), _p(x_perm), _stream(stream)))


def moe_grouped_ffn(sh, x_perm, offsets, w13, w2, y_perm, ws=None, stream=None):
    _check(lib().moe_grouped_ffn(ctypes.byref(shape_c(sh)), _p(x_perm), _p(offsets), _p(w13), _p(w2), _p(y_perm),
                                 _p(ws), 0 if ws is None else ws.numel(), _stream(stream)))


def moe_grouped_ffn_backward(sh, x_perm, offsets, w13, w2, dy_perm, dx_perm, dw13, dw2, ws=None, stream=None):
    _check(lib().moe_grouped_ffn_backward(ctypes.byref(shape_c(sh)), _p(x_perm), _p(offsets), _p(w13), _p(w2),
                                          _p(dy_perm), _p(dx_perm), _p(dw13), _p(dw2), _p(ws),
                                          0 if ws is None else ws.numel(), _stream(stream)))


def moe_layer_backward(sh, x, w_router, bias, w13, w2, ws13, ws2, dout, fwd_ws, dx, dw_router, dw13, dw2, dws13,
                       dws2, ws, stream=None):
    _check(lib().moe_layer_backward(ctypes.byref(shape_c(sh)), _p(x), _p(w_router), _p(bias), _p(w13), _p(w2),
                                    _p(ws13), _p(ws2), _p(dout), _p(fwd_ws), 0 if fwd_ws is None else fwd_ws.numel(),
                                    _p(dx), _p(dw_router), _p(dw13), _p(dw2), _p(dws13), _p(dws2), _p(ws),
                                    0 if ws is None else ws.numel(), _stream(stream)))


def moe_combine(sh, y_perm, slot_row, topk_w, shared_y, out, stream=None):
    _check(lib().moe_combine(ctypes.byref(shape_c(sh)), _p(y_perm), _p(slot_row), _p(topk_w), _p(shared_y),
                             _p(out), _stream(stream)))


def moe_layer_forward(sh, x, w_router, bias, w13, w2, ws13, ws2, out, ws, stream=None):
    _check(lib().moe_layer_forward(ctypes.byref(shape_c(sh)), _p(x), _p(w_router), _p(bias), _p(w13), _p(w2),
                                   _p(ws13), _p(ws2), _p(out), _p(ws), 0 if ws is None else ws.numel(),
                                   _stream(stream)))


def moe_layer_forward_traced(sh, x, w_router, bias, w13, w2, ws13, ws2, out, ws, events, stream=None):
    """``events``: ctypes array of len(MOE_STEP_NAMES) + 1 hipEvent_t handles (or None); a NULL
    entry is not recorded."""
    _check(lib().moe_layer_forward_traced(ctypes.byref(shape_c(sh)), _p(x), _p(w_router), _p(bias), _p(w13),
                                          _p(w2), _p(ws13), _p(ws2), _p(out), _p(ws),
                                          0 if ws is None else ws.numel(), events, _stream(stream)))


# ---------------------------------------------------------------------------------------
# block-scaled formats, the norm in front of a layer, the few-token layer
#
# These calls check their tensors (dtype, shape, contiguity, one device) before the library sees
# pointers, and run on the tensors' device, by default on its current stream.
# ---------------------------------------------------------------------------------------
def _refuse(message: str):
    raise MoEError(MOE_ERR_INVALID_ARG, message)


def _mismatch(device, name, t, dtype, wanted):
    _refuse(f"{name} is missing" if t is None else
            f"{name} is {t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}; "
            f"expected contiguous {dtype} {wanted} on {device}")


def _take(device, name, t, dtype, *shape):
    """Pointer of a tensor that has to have this dtype and shape on this device."""
    if t is None or t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        _mismatch(device, name, t, dtype, shape)
    return t.data_ptr()


def _bytes(device, name, t, n):
    """Pointer of a contiguous uint8 tensor of at least n values (any shape)."""
    if t is None or t.dtype is not _u8 or t.numel() < n or t.device != device or not t.is_contiguous():
        _mismatch(device, name, t, _u8, f"of {n} values")
    return t.data_ptr()


def _rows_of(device, name, t, rows, n):
    """Pointer of a contiguous uint8 tensor of exactly ``rows`` rows of n values: flat, or with rows as its last dimension."""
    if t is None or t.dtype is not _u8 or t.numel() != rows * n or t.device != device or not t.is_contiguous() or (
            t.dim() > 1 and t.shape[-1] != n):
        _mismatch(device, name, t, _u8, f"of {rows} rows of {n} values")
    return t.data_ptr()


def _ws(device, ws):
    """(pointer, bytes) of a workspace."""
    return (None, 0) if ws is None else (_bytes(device, "ws", ws, 0), ws.numel())


def _matrix(name, t):
    """(rows, columns, device) of a tensor on a GPU."""
    lib()
    if t.dim() != 2:
        _refuse(f"{name} has {t.dim()} dimensions, expected 2")
    if not t.is_cuda:
        _refuse(f"{name} is on {t.device}, not on a GPU")
    rows, cols = t.shape
    return rows, cols, t.device


def _on(device, stream, call, *args):
    """Runs a library call on ``device`` and ``stream`` (None: that device's current stream)."""
    index = device.index
    if stream is None:
        # the handle of torch.cuda.current_stream(device), without a Stream object (1.7 us a call)
        stream = _raw_stream(index)
    if index == _current_device():
        status = call(*args, stream)
    else:
        import torch
        with torch.cuda.device(index):
            status = call(*args, stream)
    if status != MOE_OK:
        raise MoEError(status, last_error())


def mx_elements_per_row(format: int, cols: int) -> int:
    """Bytes of one row's elements in a block-scaled format."""
    return cols // 2 if format == MOE_MX_E2M1 else cols


def moe_mx_quantize(format, x, elements, scales, stream=None):
    """bf16 ``x [rows, cols]`` into uint8 ``elements [rows, cols / 2 or cols]`` and ``scales [rows, cols / 32]``."""
    rows, cols, dev = _matrix("x", x)
    _on(dev, stream, _lib.moe_mx_quantize, rows, cols, format, _take(dev, "x", x, _bf16, rows, cols),
        _take(dev, "elements", elements, _u8, rows, mx_elements_per_row(format, cols)),
        _take(dev, "scales", scales, _u8, rows, cols // 32))


def moe_mx_dequantize(format, elements, scales, x, stream=None):
    """The values of block-scaled ``elements`` and ``scales`` into bf16 ``x [rows, cols]``."""
    rows, cols, dev = _matrix("x", x)
    _on(dev, stream, _lib.moe_mx_dequantize, rows, cols, format,
        _take(dev, "elements", elements, _u8, rows, mx_elements_per_row(format, cols)),
        _take(dev, "scales", scales, _u8, rows, cols // 32), _take(dev, "x", x, _bf16, rows, cols))


def moe_mx_grouped_ffn(sh, format, x_q, x_scales, offsets, w13_q, w13_scales, w2_q, w2_scales, y_perm, ws, stream=None):
    """The expert MLP on block-scaled rows in expert order (``format``) and e2m1 weights (flat, or rows as their last
    dimension).  ``y_perm`` has ``sh.capacity`` rows, ``x_q`` and ``x_scales`` at least as many; ``offsets`` is ``moe_permute``'s, or with an expert capacity its counts."""
    d, F, El, cap = sh.d, sh.F, sh.E_local, sh.capacity
    dev = _matrix("y_perm", y_perm)[2]
    _on(dev, stream, _lib.moe_mx_grouped_ffn, ctypes.byref(shape_c(sh)), format,
        _bytes(dev, "x_q", x_q, cap * mx_elements_per_row(format, d)), _bytes(dev, "x_scales", x_scales, cap * (d // 32)),
        _take(dev, "offsets", offsets, _i32, El if sh.expert_capacity > 0 else El + 1),
        _rows_of(dev, "w13_q", w13_q, El * 2 * F, d // 2), _rows_of(dev, "w13_scales", w13_scales, El * 2 * F, d // 32),
        _rows_of(dev, "w2_q", w2_q, El * d, F // 2), _rows_of(dev, "w2_scales", w2_scales, El * d, F // 32),
        _take(dev, "y_perm", y_perm, _bf16, cap, d), *_ws(dev, ws))


def moe_add_rmsnorm(x, residual, gamma, eps, h, y, y_q=None, y_scales=None, rstd=None, stream=None):
    """``h = x + residual``, ``y = h * rstd * gamma`` in bf16, in e4m3 blocks (``y_q``, ``y_scales``), or in both.
    Without a residual ``h`` is None; with one it may be the buffer of ``x`` or of ``residual``."""
    rows, d, dev = _matrix("x", x)
    _on(dev, stream, _lib.moe_add_rmsnorm, rows, d, eps, _take(dev, "x", x, _bf16, rows, d),
        None if residual is None else _take(dev, "residual", residual, _bf16, rows, d), _take(dev, "gamma", gamma, _bf16, d),
        None if h is None else _take(dev, "h", h, _bf16, rows, d), None if y is None else _take(dev, "y", y, _bf16, rows, d),
        None if y_q is None else _take(dev, "y_q", y_q, _u8, rows, d),
        None if y_scales is None else _take(dev, "y_scales", y_scales, _u8, rows, d // 32),
        None if rstd is None else _take(dev, "rstd", rstd, _f32, rows))


def moe_add_rmsnorm_backward(dy, dh, h, gamma, rstd, dx, dgamma, ws, stream=None):
    """``dx`` (of x and of the residual alike) and ``dgamma``; ``dh`` is the gradient that comes back to ``h``, or None.
    ``h`` and ``rstd`` are the forward's (``h`` is ``x`` where it had no residual)."""
    rows, d, dev = _matrix("dy", dy)
    _on(dev, stream, _lib.moe_add_rmsnorm_backward, rows, d, _take(dev, "dy", dy, _bf16, rows, d),
        None if dh is None else _take(dev, "dh", dh, _bf16, rows, d), _take(dev, "h", h, _bf16, rows, d),
        _take(dev, "gamma", gamma, _bf16, d), _take(dev, "rstd", rstd, _f32, rows),
        _take(dev, "dx", dx, _bf16, rows, d), _take(dev, "dgamma", dgamma, _bf16, d), *_ws(dev, ws))


def add_rmsnorm_workspace_size(rows: int, d: int) -> int:
    n = lib().moe_add_rmsnorm_workspace_size(rows, d)
    if n == 0:
        raise MoEError(MOE_ERR_INVALID_ARG, last_error())
    return n


def alloc_add_rmsnorm_workspace(rows: int, d: int, device="cuda"):
    import torch
    return torch.empty(add_rmsnorm_workspace_size(rows, d), dtype=torch.uint8, device=device)


def moe_layer_decode(sh, x, w_router, bias, w13, w2, ws13, ws2, out, ws, scales=None, stream=None):
    """The whole layer for ``sh.T <= MOE_DECODE_MAX_TOKENS`` tokens.  ``scales``: None with bf16 weights, or
    (w13_scales, w2_scales, ws13_scales, ws2_scales) with e2m1 ones (the last two None without a shared expert)."""
    T, d, F, Fs, El = sh.T, sh.d, sh.F, sh.F_shared, sh.E_local
    dev = _matrix("x", x)[2]
    s = scales if scales is not None else (None,) * 4

    def weights(name, t, s, rows, K):
        if scales is not None:
            return _rows_of(dev, name, t, rows, K // 2), _rows_of(dev, name + "_scales", s, rows, K // 32)
        if t is None or t.dtype is not _bf16 or t.numel() != rows * K or t.device != dev or not t.is_contiguous():
            _mismatch(dev, name, t, _bf16, f"of {rows * K} values")
        return t.data_ptr(), None

    none = (None, None)
    _on(dev, stream, _lib.moe_layer_decode, ctypes.byref(shape_c(sh)), _take(dev, "x", x, _bf16, T, d),
        _take(dev, "w_router", w_router, _bf16, sh.E, d), None if bias is None else _take(dev, "bias", bias, _f32, sh.E),
        *weights("w13", w13, s[0], El * 2 * F, d), *weights("w2", w2, s[1], El * d, F),
        *(weights("ws13", ws13, s[2], 2 * Fs, d) if Fs else none), *(weights("ws2", ws2, s[3], d, Fs) if Fs else none),
        _take(dev, "out", out, _bf16, T, d), *_ws(dev, ws))


# ---------------------------------------------------------------------------------------
# device placement helpers (torch is plumbing: memory and streams)
# ---------------------------------------------------------------------------------------
def to_device_bf16(bits: np.ndarray, device="cuda"):
    """uint16 bf16 bit patterns -> torch.bfloat16 device tensor (bit-exact)."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device).view(torch.bfloat16)


def bf16_bits(t) -> np.ndarray:
    """torch.bfloat16 tensor -> uint16 bit patterns on the host."""
    import torch
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class DeviceLayer:
    """Inputs of one workload resident on the GPU, with a layer workspace.

    ``forward()`` runs ``moe_layer_forward``; ``region(...)`` views the intermediates
    it left in the workspace (routing, permutation, permuted rows).
    """

    def __init__(self, inputs: dict, device="cuda"):
        import torch
        self.shape = sh = inputs["shape"]
        self.device = device
        self.x = to_device_bf16(inputs["x"], device)
        self.w_router = to_device_bf16(inputs["w_router"], device)
        self.bias = None if inputs.get("bias") is None else torch.from_numpy(inputs["bias"]).to(device)
        self.w13 = to_device_bf16(inputs["w13"], device)
        self.w2 = to_device_bf16(inputs["w2"], device)
        self.ws13 = to_device_bf16(inputs["ws13"], device) if sh.F_shared > 0 else None
        self.ws2 = to_device_bf16(inputs["ws2"], device) if sh.F_shared > 0 else None
        self.out = torch.empty((sh.T, sh.d), dtype=torch.bfloat16, device=device)
        self.ws = alloc_workspace(sh, MOE_WS_LAYER, device)

    def forward(self, stream=None):
        moe_layer_forward(self.shape, self.x, self.w_router, self.bias, self.w13, self.w2, self.ws13, self.ws2,
                          self.out, self.ws, stream)
        return self.out

    def forward_traced(self, events, stream=None):
        moe_layer_forward_traced(self.shape, self.x, self.w_router, self.bias, self.w13, self.w2, self.ws13,
                                 self.ws2, self.out, self.ws, events, stream)
        return self.out

    def backward(self, dout, stream=None):
        """``moe_layer_backward`` for output gradient ``dout`` of the last ``forward()``; returns
        the gradients as a dict of device tensors (dx, dw_router, dw13, dw2, dws13, dws2)."""
        import torch
        sh = self.shape
        dev = self.device
        bf = torch.bfloat16
        g = {"dx": torch.empty((sh.T, sh.d), dtype=bf, device=dev),
             "dw_router": torch.empty((sh.E, sh.d), dtype=bf, device=dev),
             "dw13": torch.empty((sh.E_local, 2 * sh.F, sh.d), dtype=bf, device=dev),
             "dw2": torch.empty((sh.E_local, sh.d, sh.F), dtype=bf, device=dev),
             "dws13": torch.empty((2 * sh.F_shared, sh.d), dtype=bf, device=dev) if sh.F_shared > 0 else None,
             "dws2": torch.empty((sh.d, sh.F_shared), dtype=bf, device=dev) if sh.F_shared > 0 else None}
        if getattr(self, "ws_bwd", None) is None:
            self.ws_bwd = alloc_workspace(sh, MOE_WS_LAYER_BWD, dev)
        moe_layer_backward(sh, self.x, self.w_router, self.bias, self.w13, self.w2, self.ws13, self.ws2, dout,
                           self.ws, g["dx"], g["dw_router"], g["dw13"], g["dw2"], g["dws13"], g["dws2"],
                           self.ws_bwd, stream)
        return g

    def quantize(self):
        """The expert weights in e2m1 for ``decode(mx=True)``: per tensor (elements, scales).  Called again, after the
        weights changed, it writes the same buffers, so a graph captured on them reads the new weights."""
        import torch
        held, made = getattr(self, "mx", None) or {}, {}
        for name in ("w13", "w2", "ws13", "ws2"):
            w = getattr(self, name)
            if w is not None:
                rows, cols = w.numel() // w.shape[-1], w.shape[-1]
                q, s = held[name] if name in held else (torch.empty((rows, n), dtype=torch.uint8, device=self.device)
                                                        for n in (cols // 2, cols // 32))
                moe_mx_quantize(MOE_MX_E2M1, w.view(rows, cols), q, s)
                made[name] = (q, s)
        self.mx = made
        return self.mx

    def decode(self, mx: bool = False, stream=None):
        """``moe_layer_decode`` with the layer's bf16 weights, or with the e2m1 ones of ``quantize()``."""
        if getattr(self, "ws_decode", None) is None:
            self.ws_decode = alloc_workspace(self.shape, MOE_WS_DECODE, self.device)
        names = ("w13", "w2", "ws13", "ws2")
        w, scales = [getattr(self, n) for n in names], None
        if mx:
            if getattr(self, "mx", None) is None:
                _refuse("the layer has no e2m1 weights yet: quantize() makes them")
            w, scales = zip(*(self.mx.get(n, (None, None)) for n in names))
        moe_layer_decode(self.shape, self.x, self.w_router, self.bias, *w, self.out, self.ws_decode, scales, stream)
        return self.out

    def region(self, region: int, dtype, shape):
        import torch
        off = workspace_offset(self.shape, region)
        nbytes = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        return self.ws[off:off + nbytes].view(dtype).view(*shape)
