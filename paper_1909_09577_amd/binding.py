"""Thin ctypes binding of libnmconv1d.so (C ABI: include/nm_conv1d.h).

Only argument marshalling happens here: tensors are torch device tensors whose
``data_ptr()`` is handed to the library, the stream is torch's current HIP stream,
and outputs / workspace are ``torch.empty`` buffers when the caller passes none.
Every arithmetic step runs inside the library's kernels.  If the library has not
been built, loading raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libnmconv1d.so")

NM_OK, NM_ERR_BAD_ARG, NM_ERR_UNSUPPORTED, NM_ERR_WORKSPACE, NM_ERR_DEVICE, NM_ERR_SCRATCH_LIMIT = 0, -1, -2, -3, -4, -5
NM_STATIC_SCRATCH_BYTES = 32 << 20
NM_BF16, NM_F32 = 0, 1
NM_RELU, NM_ACCUM_DW, NM_FORCE_DIRECT, NM_ACCUM_DX = 1, 2, 4, 8
NM_OP_FWD, NM_OP_BWD_DATA, NM_OP_BWD_WEIGHT, NM_OP_BWD, NM_OP_BN_FWD, NM_OP_BN_BWD = 0, 1, 2, 3, 4, 5
NM_OP_ATTN_FWD, NM_OP_ATTN_BWD = 16, 17
NM_NORM_POST, NM_NORM_NEXT, NM_NORM_LAYER = 1, 2, 4
NM_GATE_NONE, NM_GATE_ITEM, NM_GATE_ELEMENT = 0, 1, 2

EXPORTS = ("nm_conv1d_out_len", "nm_conv1d_workspace_bytes", "nm_strerror", "nm_conv1d_block_fwd",
           "nm_conv1d_bwd_data", "nm_conv1d_bwd_weight", "nm_conv1d_bwd", "nm_conv1d_block_fwd_masked", "nm_conv1d_bwd_data_masked",
           "nm_conv1d_bwd_weight_masked", "nm_decoder_logsoftmax_fwd", "nm_conv1d_block_fwd_static", "nm_conv1d_time_next_kernel_of", "nm_conv1d_bn_fwd", "nm_conv1d_bn_bwd", "nm_conv1d_bwd_masked", "nm_conv1d_time_next_main_kernel",
           "nm_conv1d_kernel_name",
           "nm_fp8_row_scales", "nm_fp8_quantize_rows", "nm_conv1d_fp8_supported", "nm_conv1d_fp8_workspace_bytes",
           "nm_conv1d_block_fwd_fp8", "nm_conv1d_bwd_data_fp8", "nm_conv1d_fp8_bwd_data_workspace_bytes",
           "nm_fp8_dgrad_weight_scales", "nm_conv1d_bwd_weight_fp8", "nm_conv1d_fp8_bwd_weight_workspace_bytes",
           "nm_conv1d_bwd_fp8", "nm_conv1d_fp8_bwd_workspace_bytes",
           "nm_cross_attn_workspace_bytes", "nm_cross_attn_fwd", "nm_cross_attn_bwd",
           "nm_residual_norm_fwd", "nm_residual_norm_bwd", "nm_residual_norm_bwd_workspace_bytes",
           "nm_adamw_plan_bytes", "nm_adamw_plan", "nm_adamw_step")

_lib = None


class AdamWTensor(ctypes.Structure):
    """nm_adamw_tensor of include/nm_adamw.h."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_longlong),
                ("weight_decay", ctypes.c_float)]


class NmError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({strerror(status)})")


def lib() -> ctypes.CDLL:
    """Load the HIP library (raises FileNotFoundError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        i, u, vp, sz = ctypes.c_int, ctypes.c_uint, ctypes.c_void_p, ctypes.c_size_t
        L.nm_conv1d_out_len.argtypes = [i] * 5
        L.nm_conv1d_out_len.restype = i
        L.nm_conv1d_workspace_bytes.argtypes = [i] * 9 + [i, u]
        L.nm_conv1d_workspace_bytes.restype = sz
        L.nm_conv1d_kernel_name.argtypes = [i] * 10 + [u, i, sz, ctypes.c_char_p, sz]
        L.nm_conv1d_kernel_name.restype = i
        L.nm_strerror.argtypes = [i]
        L.nm_strerror.restype = ctypes.c_char_p
        L.nm_conv1d_block_fwd.argtypes = [i] * 8 + [vp] * 6 + [u, i, vp, sz, vp]
        L.nm_conv1d_block_fwd.restype = i
        L.nm_conv1d_block_fwd_static.argtypes = [i] * 8 + [vp] * 6 + [u, i, vp]
        L.nm_conv1d_block_fwd_static.restype = i
        L.nm_conv1d_bwd_data.argtypes = [i] * 8 + [vp] * 6 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd_data.restype = i
        L.nm_conv1d_bwd_weight.argtypes = [i] * 8 + [vp] * 5 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd_weight.restype = i
        L.nm_conv1d_block_fwd_masked.argtypes = [i] * 8 + [vp] * 7 + [u, i, vp, sz, vp]
        L.nm_conv1d_block_fwd_masked.restype = i
        L.nm_conv1d_bwd_data_masked.argtypes = [i] * 8 + [vp] * 7 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd_data_masked.restype = i
        L.nm_conv1d_bwd_weight_masked.argtypes = [i] * 8 + [vp] * 6 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd_weight_masked.restype = i
        L.nm_conv1d_bwd.argtypes = [i] * 8 + [vp] * 8 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd.restype = i
        L.nm_conv1d_bwd_masked.argtypes = [i] * 8 + [vp] * 9 + [u, i, vp, sz, vp]
        L.nm_conv1d_bwd_masked.restype = i
        L.nm_conv1d_bn_fwd.argtypes = [i] * 8 + [vp] * 4 + [ctypes.c_float] + [vp] * 5 + [u, i, vp, sz, vp]
        L.nm_conv1d_bn_fwd.restype = i
        L.nm_conv1d_bn_bwd.argtypes = [i] * 8 + [vp] * 13 + [u, i, vp, sz, vp]
        L.nm_conv1d_bn_bwd.restype = i
        L.nm_decoder_logsoftmax_fwd.argtypes = [i] * 4 + [vp] * 4 + [u, i, vp]
        L.nm_decoder_logsoftmax_fwd.restype = i
        L.nm_conv1d_time_next_main_kernel.argtypes = [vp, vp]
        L.nm_conv1d_time_next_main_kernel.restype = i
        L.nm_conv1d_time_next_kernel_of.argtypes = [vp, vp, i]
        L.nm_conv1d_time_next_kernel_of.restype = i
        L.nm_fp8_row_scales.argtypes = [vp, i, sz, vp, vp]
        L.nm_fp8_row_scales.restype = i
        L.nm_fp8_quantize_rows.argtypes = [vp, i, sz, vp, vp, vp]
        L.nm_fp8_quantize_rows.restype = i
        L.nm_conv1d_fp8_supported.argtypes = [i] * 8
        L.nm_conv1d_fp8_supported.restype = i
        L.nm_conv1d_fp8_workspace_bytes.argtypes = [i] * 8
        L.nm_conv1d_fp8_workspace_bytes.restype = sz
        L.nm_conv1d_block_fwd_fp8.argtypes = [i] * 8 + [vp] * 8 + [u, vp, sz, vp]
        L.nm_conv1d_block_fwd_fp8.restype = i
        L.nm_conv1d_bwd_data_fp8.argtypes = [i] * 8 + [vp] * 8 + [u, vp, sz, vp]
        L.nm_conv1d_bwd_data_fp8.restype = i
        L.nm_conv1d_fp8_bwd_data_workspace_bytes.argtypes = [i] * 8
        L.nm_conv1d_fp8_bwd_data_workspace_bytes.restype = sz
        L.nm_fp8_dgrad_weight_scales.argtypes = [i] * 3 + [vp] * 4
        L.nm_fp8_dgrad_weight_scales.restype = i
        L.nm_conv1d_bwd_weight_fp8.argtypes = [i] * 8 + [vp] * 7 + [u, vp, sz, vp]
        L.nm_conv1d_bwd_weight_fp8.restype = i
        L.nm_conv1d_fp8_bwd_weight_workspace_bytes.argtypes = [i] * 8
        L.nm_conv1d_fp8_bwd_weight_workspace_bytes.restype = sz
        L.nm_conv1d_bwd_fp8.argtypes = [i] * 8 + [vp] * 11 + [u, vp, sz, vp]
        L.nm_conv1d_bwd_fp8.restype = i
        L.nm_conv1d_fp8_bwd_workspace_bytes.argtypes = [i] * 8
        L.nm_conv1d_fp8_bwd_workspace_bytes.restype = sz
        ll, f, d = ctypes.c_longlong, ctypes.c_float, ctypes.c_double
        L.nm_cross_attn_workspace_bytes.argtypes = [i] * 8
        L.nm_cross_attn_workspace_bytes.restype = sz
        L.nm_cross_attn_fwd.argtypes = [i] * 6 + [vp, ll] * 3 + [vp] * 3 + [f, vp, ll, vp, i, vp, sz, vp]
        L.nm_cross_attn_fwd.restype = i
        L.nm_cross_attn_bwd.argtypes = [i] * 6 + [vp, ll] * 5 + [vp] * 4 + [f] + [vp, ll] * 3 + [i, vp, sz, vp]
        L.nm_cross_attn_bwd.restype = i
        L.nm_residual_norm_fwd.argtypes = [i] * 3 + [vp] * 3 + [i] + [vp] * 5 + [f] + [vp] * 3 + [u, i, vp]
        L.nm_residual_norm_fwd.restype = i
        L.nm_residual_norm_bwd_workspace_bytes.argtypes = [i] * 4
        L.nm_residual_norm_bwd_workspace_bytes.restype = sz
        L.nm_residual_norm_bwd.argtypes = [i] * 3 + [vp] * 5 + [i] + [vp] * 4 + [f] + [vp] * 9 + [u, i, vp, sz, vp]
        L.nm_residual_norm_bwd.restype = i
        L.nm_adamw_plan_bytes.argtypes = [ctypes.POINTER(AdamWTensor), i, i]
        L.nm_adamw_plan_bytes.restype = sz
        L.nm_adamw_plan.argtypes = [ctypes.POINTER(AdamWTensor), i, i, vp, sz]
        L.nm_adamw_plan.restype = i
        L.nm_adamw_step.argtypes = [vp, vp, sz, d, d, d, d, ll, vp, u, vp]
        L.nm_adamw_step.restype = i
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().nm_strerror(int(status)).decode()


def nm_conv1d_out_len(T: int, K: int, stride: int = 1, dilation: int = 1, pad: int = 0) -> int:
    return int(lib().nm_conv1d_out_len(T, K, stride, dilation, pad))


def nm_conv1d_workspace_bytes(op: int, B, Cin, Cout, T, K, stride=1, dilation=1, pad=0, dtype=NM_BF16,
                              flags=0) -> int:
    return int(lib().nm_conv1d_workspace_bytes(op, B, Cin, Cout, T, K, stride, dilation, pad, dtype, flags))


def nm_conv1d_kernel_name(op: int, B, Cin, Cout, T, K, stride=1, dilation=1, pad=0, dtype=NM_BF16, flags=0, masked=False,
                          workspace_bytes=None) -> str:
    """Name of the main kernel of a pass (workspace_bytes None: of the size asked for)."""
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    if workspace_bytes is None:
        workspace_bytes = nm_conv1d_workspace_bytes(NM_OP_FWD if op == NM_OP_BN_FWD else op, *dims, dtype, flags)
    name = ctypes.create_string_buffer(128)
    st = lib().nm_conv1d_kernel_name(op, *dims, dtype, flags, 1 if masked else 0, workspace_bytes, name, len(name))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_kernel_name")
    return name.value.decode()


def nm_conv1d_time_next_main_kernel(start_event, stop_event) -> None:
    """Arm the one-shot timer with two torch.cuda.Event(enable_timing=True) objects that have
    been recorded at least once (torch creates the underlying handle lazily), or None to disarm."""
    if start_event is None or stop_event is None:
        lib().nm_conv1d_time_next_main_kernel(None, None)
        return
    lib().nm_conv1d_time_next_main_kernel(ctypes.c_void_p(start_event.cuda_event), ctypes.c_void_p(stop_event.cuda_event))


def nm_conv1d_time_next_kernel_of(start_event, stop_event, op: int) -> None:
    """Like nm_conv1d_time_next_main_kernel for the main kernel of pass `op` (NM_OP_FWD / _BWD_DATA / _BWD_WEIGHT)."""
    st = lib().nm_conv1d_time_next_kernel_of(ctypes.c_void_p(start_event.cuda_event), ctypes.c_void_p(stop_event.cuda_event),
                                             int(op))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_time_next_kernel_of")


# ---- tensor marshalling -----------------------------------------------------------------
# A call of one short utterance is over on the device in about the time that Python takes to make it, so what happens here
# per tensor counts: plain integers for pointers (the argument types convert them), shapes compared as they are, the
# stream's handle without a Stream object, no workspace query where the caller brings one.  256 channels, K=11, 200 steps,
# six tensors: 17.6 -> 13.2 us a call.
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return NM_BF16
    if t.dtype == torch.float32:
        return NM_F32
    raise TypeError(f"unsupported storage dtype {t.dtype}")


def _ptr(t, dtype=None, shape=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    c = _torch()._C
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())  # what torch.cuda.current_stream().cuda_stream says


def _out_len(T, K, stride, dilation, pad):
    """nm_conv1d_out_len; plain cases without the call."""
    span = T + 2 * pad - dilation * (K - 1) - 1
    if 0 <= span < 1 << 30 and T > 0 and K > 0 and stride > 0 and dilation > 0 and pad >= 0:
        return span // stride + 1
    return nm_conv1d_out_len(T, K, stride, dilation, pad)


def _workspace(op, dims, dtype_code, flags, workspace, like):
    if workspace is None:
        need = nm_conv1d_workspace_bytes(op, *dims, dtype_code, flags)
        workspace = like.new_empty(max(need, 256), dtype=_torch().uint8)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def nm_conv1d_block_fwd(x, w, scale=None, shift=None, residual=None, y=None, *, stride=1, dilation=1,
                        pad=0, relu=False, force_direct=False, workspace=None, stream=None, lengths=None):
    """y = relu?(scale*conv1d(x,w)+shift+residual); returns y (allocated if not given).
    lengths (int32 [B], optional): valid length of every sample, the rest of x reads as zero."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = _out_len(T, K, stride, dilation, pad)
    if To <= 0:
        raise NmError(NM_ERR_BAD_ARG, "nm_conv1d_block_fwd")
    code = _dtype_code(x)
    if y is None:
        y = x.new_empty((B, Cout, To))
    flags = (NM_RELU if relu else 0) | (NM_FORCE_DIRECT if force_direct else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_FWD, dims, code, flags, workspace, x)
    fn, extra = (lib().nm_conv1d_block_fwd, ()) if lengths is None else (
        lib().nm_conv1d_block_fwd_masked, (_ptr(lengths, torch.int32, (B,), "lengths"),))
    st = fn(
        *dims, *extra, _ptr(x, name="x"), _ptr(w, x.dtype, (Cout, Cin, K), "w"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(shift, torch.float32, (Cout,), "shift"),
        _ptr(residual, x.dtype, (B, Cout, To), "residual"), _ptr(y, x.dtype, (B, Cout, To), "y"),
        flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_block_fwd")
    return y


def nm_conv1d_block_fwd_static(x, w, scale=None, shift=None, residual=None, *, y, stride=1, dilation=1, pad=0,
                               relu=False, force_direct=False, stream=None):
    """nm_conv1d_block_fwd without a workspace: scratch is the library's fixed array.  The caller passes
    the output tensor y (this wrapper allocates nothing either); returns y."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = y.shape[2]
    flags = (NM_RELU if relu else 0) | (NM_FORCE_DIRECT if force_direct else 0)
    st = lib().nm_conv1d_block_fwd_static(
        B, Cin, Cout, T, K, stride, dilation, pad, _ptr(x, name="x"), _ptr(w, x.dtype, (Cout, Cin, K), "w"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(shift, torch.float32, (Cout,), "shift"),
        _ptr(residual, x.dtype, (B, Cout, To), "residual"), _ptr(y, x.dtype, (B, Cout, To), "y"),
        flags, _dtype_code(x), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_block_fwd_static")
    return y


def nm_conv1d_bwd_data(dy, w, T, y=None, scale=None, dx=None, dres=None, *, stride=1, dilation=1, pad=0,
                       relu=False, want_dres=False, force_direct=False, workspace=None, stream=None, lengths=None,
                       accumulate_dx=False):
    """dx (and optionally dres) from the upstream gradient dy; returns (dx, dres).
    lengths (int32 [B], optional): valid input length of every sample; dx is zero beyond it."""
    torch = _torch()
    B, Cout, To = dy.shape
    _, Cin, K = w.shape
    code = _dtype_code(dy)
    if dx is None:
        if accumulate_dx:
            raise ValueError("accumulate_dx needs an existing dx")
        dx = torch.empty((B, Cin, T), dtype=dy.dtype, device=dy.device)
    if dres is None and want_dres:
        dres = torch.empty_like(dy)
    flags = (NM_RELU if relu else 0) | (NM_FORCE_DIRECT if force_direct else 0) | (NM_ACCUM_DX if accumulate_dx else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_BWD_DATA, dims, code, flags, workspace, dy)
    fn, extra = (lib().nm_conv1d_bwd_data, ()) if lengths is None else (
        lib().nm_conv1d_bwd_data_masked, (_ptr(lengths, torch.int32, (B,), "lengths"),))
    st = fn(
        *dims, *extra, _ptr(dy, name="dy"), _ptr(y, dy.dtype, (B, Cout, To), "y"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(w, dy.dtype, (Cout, Cin, K), "w"),
        _ptr(dx, dy.dtype, (B, Cin, T), "dx"), _ptr(dres, dy.dtype, (B, Cout, To), "dres"),
        flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd_data")
    return dx, dres


def nm_conv1d_bwd_weight(x, dy, K, y=None, scale=None, dw=None, *, stride=1, dilation=1, pad=0,
                         relu=False, accumulate=False, force_direct=False, workspace=None, stream=None, lengths=None):
    """dw [Cout,Cin,K] float32 from x and the upstream gradient dy; returns dw.
    lengths (int32 [B], optional): valid length of every sample, the rest of x reads as zero."""
    torch = _torch()
    B, Cin, T = x.shape
    _, Cout, To = dy.shape
    code = _dtype_code(x)
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs an existing dw")
        dw = torch.empty((Cout, Cin, K), dtype=torch.float32, device=x.device)
    flags = (NM_RELU if relu else 0) | (NM_ACCUM_DW if accumulate else 0) | (NM_FORCE_DIRECT if force_direct else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_BWD_WEIGHT, dims, code, flags, workspace, x)
    fn, extra = (lib().nm_conv1d_bwd_weight, ()) if lengths is None else (
        lib().nm_conv1d_bwd_weight_masked, (_ptr(lengths, torch.int32, (B,), "lengths"),))
    st = fn(
        *dims, *extra, _ptr(x, name="x"), _ptr(dy, x.dtype, (B, Cout, To), "dy"), _ptr(y, x.dtype, (B, Cout, To), "y"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(dw, torch.float32, (Cout, Cin, K), "dw"),
        flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd_weight")
    return dw


def nm_conv1d_bwd(x, dy, w, y=None, scale=None, dx=None, dres=None, dw=None, *, stride=1, dilation=1, pad=0,
                  relu=False, want_dres=False, accumulate=False, force_direct=False, workspace=None, stream=None,
                  accumulate_dx=False, lengths=None):
    """Both gradients in one call; returns (dx, dres, dw).  lengths (int32 [B], optional): padded batch."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = dy.shape[2]
    code = _dtype_code(x)
    if dx is None:
        if accumulate_dx:
            raise ValueError("accumulate_dx needs an existing dx")
        dx = torch.empty((B, Cin, T), dtype=x.dtype, device=x.device)
    if dres is None and want_dres:
        dres = torch.empty_like(dy)
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs an existing dw")
        dw = torch.empty((Cout, Cin, K), dtype=torch.float32, device=x.device)
    flags = (NM_RELU if relu else 0) | (NM_ACCUM_DW if accumulate else 0) | (NM_FORCE_DIRECT if force_direct else 0) | \
        (NM_ACCUM_DX if accumulate_dx else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_BWD, dims, code, flags, workspace, x)
    fn, extra = (lib().nm_conv1d_bwd, ()) if lengths is None else (
        lib().nm_conv1d_bwd_masked, (_ptr(lengths, torch.int32, (B,), "lengths"),))
    st = fn(
        *dims, *extra, _ptr(x, name="x"), _ptr(dy, x.dtype, (B, Cout, To), "dy"), _ptr(y, x.dtype, (B, Cout, To), "y"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(w, x.dtype, (Cout, Cin, K), "w"),
        _ptr(dx, x.dtype, (B, Cin, T), "dx"), _ptr(dres, x.dtype, (B, Cout, To), "dres"),
        _ptr(dw, torch.float32, (Cout, Cin, K), "dw"), flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd")
    return dx, dres, dw


def nm_conv1d_bn_fwd(x, w, gamma=None, beta=None, residual=None, *, eps=1e-3, stride=1, dilation=1, pad=0, relu=False,
                     force_direct=False, z=None, y=None, mean=None, invstd=None, workspace=None, stream=None):
    """Block forward with training-mode BatchNorm; returns (z, y, mean, invstd)."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = _out_len(T, K, stride, dilation, pad)
    if To <= 0:
        raise NmError(NM_ERR_BAD_ARG, "nm_conv1d_bn_fwd")
    code = _dtype_code(x)
    z = torch.empty((B, Cout, To), dtype=x.dtype, device=x.device) if z is None else z
    y = torch.empty((B, Cout, To), dtype=x.dtype, device=x.device) if y is None else y
    mean = torch.empty((Cout,), dtype=torch.float32, device=x.device) if mean is None else mean
    invstd = torch.empty((Cout,), dtype=torch.float32, device=x.device) if invstd is None else invstd
    flags = (NM_RELU if relu else 0) | (NM_FORCE_DIRECT if force_direct else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_BN_FWD, dims, code, flags, workspace, x)
    st = lib().nm_conv1d_bn_fwd(
        *dims, _ptr(x, name="x"), _ptr(w, x.dtype, (Cout, Cin, K), "w"), _ptr(gamma, torch.float32, (Cout,), "gamma"),
        _ptr(beta, torch.float32, (Cout,), "beta"), float(eps), _ptr(residual, x.dtype, (B, Cout, To), "residual"),
        _ptr(z, x.dtype, (B, Cout, To), "z"), _ptr(y, x.dtype, (B, Cout, To), "y"), _ptr(mean, torch.float32, (Cout,), "mean"),
        _ptr(invstd, torch.float32, (Cout,), "invstd"), flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bn_fwd")
    return z, y, mean, invstd


def nm_conv1d_bn_bwd(x, w, gamma, z, y, mean, invstd, dy, *, stride=1, dilation=1, pad=0, relu=False, want_dres=False,
                     force_direct=False, accumulate=False, accumulate_dx=False, dx=None, dres=None, dw=None, dgamma=None,
                     dbeta=None, workspace=None, stream=None):
    """Backward of nm_conv1d_bn_fwd; returns (dx, dres, dw, dgamma, dbeta)."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = dy.shape[2]
    code = _dtype_code(x)
    if (accumulate and (dw is None or dgamma is None or dbeta is None)) or (accumulate_dx and dx is None):
        raise ValueError("accumulation needs existing output tensors")
    dx = torch.empty((B, Cin, T), dtype=x.dtype, device=x.device) if dx is None else dx
    if dres is None and want_dres:
        dres = torch.empty_like(dy)
    dw = torch.empty((Cout, Cin, K), dtype=torch.float32, device=x.device) if dw is None else dw
    dgamma = torch.empty((Cout,), dtype=torch.float32, device=x.device) if dgamma is None else dgamma
    dbeta = torch.empty((Cout,), dtype=torch.float32, device=x.device) if dbeta is None else dbeta
    flags = (NM_RELU if relu else 0) | (NM_ACCUM_DW if accumulate else 0) | (NM_FORCE_DIRECT if force_direct else 0) | \
        (NM_ACCUM_DX if accumulate_dx else 0)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    ws, ws_ptr, ws_bytes = _workspace(NM_OP_BN_BWD, dims, code, flags, workspace, x)
    act = (B, Cout, To)
    st = lib().nm_conv1d_bn_bwd(
        *dims, _ptr(x, name="x"), _ptr(w, x.dtype, (Cout, Cin, K), "w"), _ptr(gamma, torch.float32, (Cout,), "gamma"),
        _ptr(z, x.dtype, act, "z"), _ptr(y, x.dtype, act, "y"), _ptr(mean, torch.float32, (Cout,), "mean"),
        _ptr(invstd, torch.float32, (Cout,), "invstd"), _ptr(dy, x.dtype, act, "dy"), _ptr(dx, x.dtype, (B, Cin, T), "dx"),
        _ptr(dres, x.dtype, act, "dres"), _ptr(dw, torch.float32, (Cout, Cin, K), "dw"),
        _ptr(dgamma, torch.float32, (Cout,), "dgamma"), _ptr(dbeta, torch.float32, (Cout,), "dbeta"),
        flags, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bn_bwd")
    return dx, dres, dw, dgamma, dbeta


def nm_decoder_logsoftmax_fwd(x, w, bias=None, logp=None, *, force_direct=False, stream=None):
    """logp [B,Ncls,T] float32 = log_softmax over classes of (w @ x + bias); w is [Ncls,Cin]."""
    torch = _torch()
    B, Cin, T = x.shape
    Ncls = w.shape[0]
    code = _dtype_code(x)
    if logp is None:
        logp = torch.empty((B, Ncls, T), dtype=torch.float32, device=x.device)
    st = lib().nm_decoder_logsoftmax_fwd(
        B, Cin, Ncls, T, _ptr(x, name="x"), _ptr(w, x.dtype, (Ncls, Cin), "w"), _ptr(bias, torch.float32, (Ncls,), "bias"),
        _ptr(logp, torch.float32, (B, Ncls, T), "logp"), NM_FORCE_DIRECT if force_direct else 0, code, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_decoder_logsoftmax_fwd")
    return logp


# ---- 8-bit floating-point (E4M3) variant of the block forward (include/nm_conv1d_fp8.h) ------------------
def nm_fp8_row_scales(x, rows: int, *, stream=None):
    """float32 [rows]: amax/448 of each of `rows` equal slices of the bfloat16 tensor x (1 for an all-zero slice)."""
    torch = _torch()
    if x.dtype != torch.bfloat16:
        raise TypeError("x must be bfloat16")
    n = x.numel()
    if rows <= 0 or n % rows:
        raise ValueError("rows must divide the number of elements")
    scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    st = lib().nm_fp8_row_scales(_ptr(x, name="x"), rows, n // rows, _ptr(scales), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_fp8_row_scales")
    return scales


def nm_fp8_quantize_rows(x, scales, *, stream=None):
    """uint8 tensor shaped like x: the E4M3 codes of x with slice r divided by scales[r]."""
    torch = _torch()
    if x.dtype != torch.bfloat16:
        raise TypeError("x must be bfloat16")
    rows = scales.numel()
    n = x.numel()
    if rows <= 0 or n % rows:
        raise ValueError("len(scales) must divide the number of elements")
    codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    st = lib().nm_fp8_quantize_rows(_ptr(x, name="x"), rows, n // rows, _ptr(scales, torch.float32, (rows,), "scales"),
                                    _ptr(codes), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_fp8_quantize_rows")
    return codes


def nm_conv1d_fp8_supported(B, Cin, Cout, T, K, stride=1, dilation=1, pad=0) -> bool:
    return bool(lib().nm_conv1d_fp8_supported(B, Cin, Cout, T, K, stride, dilation, pad))


def nm_conv1d_fp8_workspace_bytes(B, Cin, Cout, T, K, stride=1, dilation=1, pad=0) -> int:
    return int(lib().nm_conv1d_fp8_workspace_bytes(B, Cin, Cout, T, K, stride, dilation, pad))


def nm_conv1d_block_fwd_fp8(x, x_scale, w, w_scales, scale=None, shift=None, residual=None, y=None, *, stride=1,
                            dilation=1, pad=0, relu=False, workspace=None, stream=None):
    """Block forward on E4M3 operands: x and w (bfloat16) are quantised inside the call with x_scale [1] and
    w_scales [Cout] (float32 device tensors); returns y (bfloat16, allocated if not given)."""
    torch = _torch()
    B, Cin, T = x.shape
    Cout, _, K = w.shape
    To = _out_len(T, K, stride, dilation, pad)
    if To <= 0:
        raise NmError(NM_ERR_BAD_ARG, "nm_conv1d_block_fwd_fp8")
    if y is None:
        y = torch.empty((B, Cout, To), dtype=torch.bfloat16, device=x.device)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    if workspace is None:
        workspace = torch.empty(max(nm_conv1d_fp8_workspace_bytes(*dims), 256), dtype=torch.uint8, device=x.device)
    st = lib().nm_conv1d_block_fwd_fp8(
        *dims, _ptr(x, torch.bfloat16, name="x"), _ptr(x_scale, torch.float32, (1,), "x_scale"),
        _ptr(w, torch.bfloat16, (Cout, Cin, K), "w"), _ptr(w_scales, torch.float32, (Cout,), "w_scales"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(shift, torch.float32, (Cout,), "shift"),
        _ptr(residual, torch.bfloat16, (B, Cout, To), "residual"), _ptr(y, torch.bfloat16, (B, Cout, To), "y"),
        NM_RELU if relu else 0, workspace.data_ptr(), workspace.numel(), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_block_fwd_fp8")
    return y


def nm_fp8_dgrad_weight_scales(w, scale=None, *, stream=None):
    """float32 [Cin]: per-input-channel scales of the input gradient's weight operand w[co,ci,k]*scale[co]."""
    torch = _torch()
    Cout, Cin, K = w.shape
    out = torch.empty(Cin, dtype=torch.float32, device=w.device)
    st = lib().nm_fp8_dgrad_weight_scales(Cin, Cout, K, _ptr(w, torch.bfloat16, name="w"),
                                          _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(out), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_fp8_dgrad_weight_scales")
    return out


def nm_conv1d_fp8_bwd_data_workspace_bytes(B, Cin, Cout, T, K, stride=1, dilation=1, pad=0) -> int:
    return int(lib().nm_conv1d_fp8_bwd_data_workspace_bytes(B, Cin, Cout, T, K, stride, dilation, pad))


def nm_conv1d_bwd_data_fp8(dy, g_scale, w, wt_scales, T, y=None, scale=None, dx=None, dres=None, *, stride=1, dilation=1,
                           pad=0, relu=False, want_dres=False, workspace=None, stream=None):
    """Input gradient on E4M3 operands; returns (dx, dres)."""
    torch = _torch()
    B, Cout, To = dy.shape
    _, Cin, K = w.shape
    if dx is None:
        dx = torch.empty((B, Cin, T), dtype=torch.bfloat16, device=dy.device)
    if dres is None and want_dres:
        dres = torch.empty_like(dy)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    if workspace is None:
        workspace = torch.empty(max(nm_conv1d_fp8_bwd_data_workspace_bytes(*dims), 256), dtype=torch.uint8, device=dy.device)
    st = lib().nm_conv1d_bwd_data_fp8(
        *dims, _ptr(dy, torch.bfloat16, name="dy"), _ptr(y, torch.bfloat16, (B, Cout, To), "y"),
        _ptr(g_scale, torch.float32, (1,), "g_scale"), _ptr(w, torch.bfloat16, (Cout, Cin, K), "w"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(wt_scales, torch.float32, (Cin,), "wt_scales"),
        _ptr(dx, torch.bfloat16, (B, Cin, T), "dx"), _ptr(dres, torch.bfloat16, (B, Cout, To), "dres"),
        NM_RELU if relu else 0, workspace.data_ptr(), workspace.numel(), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd_data_fp8")
    return dx, dres


def nm_conv1d_fp8_bwd_weight_workspace_bytes(B, Cin, Cout, T, K, stride=1, dilation=1, pad=0) -> int:
    return int(lib().nm_conv1d_fp8_bwd_weight_workspace_bytes(B, Cin, Cout, T, K, stride, dilation, pad))


def nm_conv1d_bwd_weight_fp8(x, x_scale, dy, g_scale, K, y=None, scale=None, dw=None, *, stride=1, dilation=1, pad=0,
                             relu=False, accumulate=False, workspace=None, stream=None):
    """Weight gradient on E4M3 operands; returns dw [Cout, Cin, K] float32."""
    torch = _torch()
    B, Cin, T = x.shape
    _, Cout, To = dy.shape
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs an existing dw")
        dw = torch.empty((Cout, Cin, K), dtype=torch.float32, device=x.device)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    if workspace is None:
        workspace = torch.empty(max(nm_conv1d_fp8_bwd_weight_workspace_bytes(*dims), 256), dtype=torch.uint8, device=x.device)
    flags = (NM_RELU if relu else 0) | (NM_ACCUM_DW if accumulate else 0)
    st = lib().nm_conv1d_bwd_weight_fp8(
        *dims, _ptr(x, torch.bfloat16, name="x"), _ptr(x_scale, torch.float32, (1,), "x_scale"),
        _ptr(dy, torch.bfloat16, name="dy"), _ptr(y, torch.bfloat16, (B, Cout, To), "y"),
        _ptr(g_scale, torch.float32, (1,), "g_scale"), _ptr(scale, torch.float32, (Cout,), "scale"),
        _ptr(dw, torch.float32, (Cout, Cin, K), "dw"), flags, workspace.data_ptr(), workspace.numel(),
        _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd_weight_fp8")
    return dw


def nm_conv1d_fp8_bwd_workspace_bytes(B, Cin, Cout, T, K, stride=1, dilation=1, pad=0) -> int:
    return int(lib().nm_conv1d_fp8_bwd_workspace_bytes(B, Cin, Cout, T, K, stride, dilation, pad))


def nm_conv1d_bwd_fp8(x, x_scale, dy, g_scale, w, wt_scales, y=None, scale=None, dx=None, dres=None, dw=None, *, stride=1,
                      dilation=1, pad=0, relu=False, want_dres=False, accumulate=False, workspace=None, stream=None):
    """Both gradients on E4M3 operands from one call; returns (dx, dres, dw)."""
    torch = _torch()
    B, Cin, T = x.shape
    _, Cout, To = dy.shape
    K = w.shape[2]
    if dx is None:
        dx = torch.empty_like(x)
    if dres is None and want_dres:
        dres = torch.empty_like(dy)
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs an existing dw")
        dw = torch.empty((Cout, Cin, K), dtype=torch.float32, device=x.device)
    dims = (B, Cin, Cout, T, K, stride, dilation, pad)
    if workspace is None:
        workspace = torch.empty(max(nm_conv1d_fp8_bwd_workspace_bytes(*dims), 256), dtype=torch.uint8, device=x.device)
    flags = (NM_RELU if relu else 0) | (NM_ACCUM_DW if accumulate else 0)
    st = lib().nm_conv1d_bwd_fp8(
        *dims, _ptr(x, torch.bfloat16, name="x"), _ptr(x_scale, torch.float32, (1,), "x_scale"),
        _ptr(dy, torch.bfloat16, name="dy"), _ptr(y, torch.bfloat16, (B, Cout, To), "y"),
        _ptr(g_scale, torch.float32, (1,), "g_scale"), _ptr(w, torch.bfloat16, (Cout, Cin, K), "w"),
        _ptr(scale, torch.float32, (Cout,), "scale"), _ptr(wt_scales, torch.float32, (Cin,), "wt_scales"),
        _ptr(dx, torch.bfloat16, (B, Cin, T), "dx"), _ptr(dres, torch.bfloat16, (B, Cout, To), "dres"),
        _ptr(dw, torch.float32, (Cout, Cin, K), "dw"), flags, workspace.data_ptr(), workspace.numel(),
        _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_conv1d_bwd_fp8")
    return dx, dres, dw


# ---- cross attention (include/nm_attention.h) ---------------------------------------------------
def _item_ptr(t, dtype, shape, name):
    """(pointer, distance of the batch items) of a tensor whose items are dense."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    B, C, N = shape
    if t.is_contiguous():
        return t.data_ptr(), C * N
    step, rows, cols = t.stride()
    if (N > 1 and cols != 1) or (C > 1 and rows != N):
        raise ValueError(f"{name} must have dense items [channels][positions]")
    if B == 1:
        step = C * N
    if step < C * N:
        raise ValueError(f"the items of {name} must not overlap")
    return t.data_ptr(), step


@functools.lru_cache(maxsize=1024)
def nm_cross_attn_workspace_bytes(op: int, B, heads, kv_heads, D, U, T, dtype=NM_BF16) -> int:
    return int(lib().nm_cross_attn_workspace_bytes(op, B, heads, kv_heads, D, U, T, dtype))


def _attn_dims(q, k, heads, kv_heads, where):
    kv_heads = heads if kv_heads is None else kv_heads
    if q.dim() != 3 or k.dim() != 3 or heads <= 0 or kv_heads <= 0 or q.shape[1] % heads:
        raise NmError(NM_ERR_BAD_ARG, where)
    B, HD, U = q.shape
    return B, heads, kv_heads, HD // heads, U, k.shape[2]


def _attn_workspace(op, dims, code, workspace, like, stream):
    if workspace is None:
        need = nm_cross_attn_workspace_bytes(op, *dims, code)
        if not need:
            return None, None, 0
        workspace = like.new_empty(need, dtype=_torch().uint8)
        if stream is not None:
            workspace.record_stream(stream)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def nm_cross_attn_fwd(q, k, v, *, heads, kv_heads=None, scale=None, lengths=None, q_lengths=None, windows=None, o=None,
                      lse=None, want_lse=False, workspace=None, stream=None):
    """Attention of the tokens q [B, heads*D, U] to the states k, v [B, kv_heads*D, T]; returns (o, lse), lse None unless given
    or wanted.  scale: 1/sqrt(D) if None.  lengths, q_lengths int32 [B]: valid states and tokens of every item; windows int32
    [B, U, 2]: first state and end of the states that a token looks at."""
    torch = _torch()
    dims = B, H, Hkv, D, U, T = _attn_dims(q, k, heads, kv_heads, "nm_cross_attn_fwd")
    code = _dtype_code(q)
    qp, qs = _item_ptr(q, q.dtype, (B, H * D, U), "q")
    kp, ks = _item_ptr(k, q.dtype, (B, Hkv * D, T), "k")
    vp, vs = _item_ptr(v, q.dtype, (B, Hkv * D, T), "v")
    if o is None:
        o = q.new_empty((B, H * D, U))
    op, os_ = _item_ptr(o, q.dtype, (B, H * D, U), "o")
    if lse is None and want_lse:
        lse = q.new_empty((B, H, U), dtype=torch.float32)
    ws, ws_ptr, ws_bytes = _attn_workspace(NM_OP_ATTN_FWD, dims, code, workspace, q, stream)
    st = lib().nm_cross_attn_fwd(
        *dims, qp, qs, kp, ks, vp, vs, _ptr(lengths, torch.int32, (B,), "lengths"),
        _ptr(q_lengths, torch.int32, (B,), "q_lengths"), _ptr(windows, torch.int32, (B, U, 2), "windows"),
        D ** -0.5 if scale is None else scale, op, os_, _ptr(lse, torch.float32, (B, H, U), "lse"), code, ws_ptr, ws_bytes,
        _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_cross_attn_fwd")
    return o, lse


def nm_cross_attn_bwd(do, q, k, v, o, lse, *, heads, kv_heads=None, scale=None, lengths=None, q_lengths=None, windows=None,
                      dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Gradients (dq, dk, dv) from the gradient do of o; o, lse and the other arguments as of the forward call."""
    torch = _torch()
    dims = B, H, Hkv, D, U, T = _attn_dims(q, k, heads, kv_heads, "nm_cross_attn_bwd")
    code = _dtype_code(q)
    q_shape, kv_shape = (B, H * D, U), (B, Hkv * D, T)
    dq = q.new_empty(q_shape) if dq is None else dq
    dk = q.new_empty(kv_shape) if dk is None else dk
    dv = q.new_empty(kv_shape) if dv is None else dv
    ins = [a for t, shape, name in ((do, q_shape, "do"), (q, q_shape, "q"), (k, kv_shape, "k"), (v, kv_shape, "v"), (o, q_shape, "o"))
           for a in _item_ptr(t, q.dtype, shape, name)]
    outs = [a for t, shape, name in ((dq, q_shape, "dq"), (dk, kv_shape, "dk"), (dv, kv_shape, "dv"))
            for a in _item_ptr(t, q.dtype, shape, name)]
    ws, ws_ptr, ws_bytes = _attn_workspace(NM_OP_ATTN_BWD, dims, code, workspace, q, stream)
    st = lib().nm_cross_attn_bwd(
        *dims, *ins, _ptr(lse, torch.float32, (B, H, U), "lse"), _ptr(lengths, torch.int32, (B,), "lengths"),
        _ptr(q_lengths, torch.int32, (B,), "q_lengths"), _ptr(windows, torch.int32, (B, U, 2), "windows"),
        D ** -0.5 if scale is None else scale, *outs, code, ws_ptr, ws_bytes, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_cross_attn_bwd")
    return dq, dk, dv


# ---- norms around a block (include/nm_norm.h) ---------------------------------------------------
def _gate_kind(gate, like, name="gate"):
    """(kind, pointer) of a gate: None, [B, C] float32 or [B, C, T] in the storage dtype."""
    B, C, T = like.shape
    if gate is None:
        return NM_GATE_NONE, None
    if gate.dim() == 2:
        return NM_GATE_ITEM, _ptr(gate, _torch().float32, (B, C), name)
    return NM_GATE_ELEMENT, _ptr(gate, like.dtype, (B, C, T), name)


def nm_residual_norm_fwd(x, f=None, *, gate=None, rscale=None, post_norm=None, post_weight=None, post_bias=None, next_norm=True,
                         next_weight=None, next_bias=None, layer=False, eps=1e-5, lengths=None, y=None, n=None, stream=None):
    """y = x + rscale*gate*h with h = f or its norm, n = norm(y); returns (y, n).  Without f: (x, norm(x)).
    post_norm: whether f is normalised (None: if post_weight is given); next_norm: whether n is made (else None);
    layer: LayerNorm instead of RMS norm.  lengths int32 [B]: zeros beyond."""
    torch = _torch()
    B, C, T = x.shape
    post = (post_weight is not None) if post_norm is None else bool(post_norm)
    if f is not None and y is None:
        y = torch.empty_like(x)
    if next_norm and n is None:
        n = torch.empty_like(x)
    kind, gp = _gate_kind(gate, x)
    flags = (NM_NORM_POST if post else 0) | (NM_NORM_NEXT if next_norm else 0) | (NM_NORM_LAYER if layer else 0)
    dt, f32, all_, c = x.dtype, torch.float32, x.shape, (C,)
    st = lib().nm_residual_norm_fwd(
        B, C, T, _ptr(x, name="x"), _ptr(f, dt, all_, "f"), gp, kind, _ptr(rscale, f32, c, "rscale"),
        _ptr(post_weight, f32, c, "post_weight"), _ptr(post_bias, f32, c, "post_bias"), _ptr(next_weight, f32, c, "next_weight"),
        _ptr(next_bias, f32, c, "next_bias"), eps, _ptr(lengths, torch.int32, (B,), "lengths"), _ptr(y, dt, all_, "y"),
        _ptr(n, dt, all_, "n"), flags, _dtype_code(x), _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_residual_norm_fwd")
    return (x if f is None else y), n


@functools.lru_cache(maxsize=1024)
def nm_residual_norm_bwd_workspace_bytes(B, C, T, dtype=NM_BF16) -> int:
    return int(lib().nm_residual_norm_bwd_workspace_bytes(B, C, T, dtype))


def nm_residual_norm_bwd(dy, dn, y, f=None, *, gate=None, rscale=None, post_norm=None, post_weight=None, post_bias=None,
                         next_weight=None, next_bias=None, layer=False, eps=1e-5, lengths=None, out=None, workspace=None,
                         stream=None):
    """Gradients of nm_residual_norm_fwd from dy (or None) and dn (None: there was no next norm): a dict with dx, df, dgate, drscale,
    dpost_weight, dpost_bias, dnext_weight, dnext_bias, None where there is nothing to differentiate.  y as the forward call
    returned it.  Gradients of vectors are made for those that are given (float32); out: a dict of tensors to write them to."""
    torch = _torch()
    like = dn if dy is None else dy
    if like is None:
        raise NmError(NM_ERR_BAD_ARG, "nm_residual_norm_bwd")
    B, C, T = like.shape
    post = (post_weight is not None) if post_norm is None else bool(post_norm)
    kind, gp = _gate_kind(gate, like)
    flags = (NM_NORM_POST if post else 0) | (NM_NORM_NEXT if dn is not None else 0) | (NM_NORM_LAYER if layer else 0)
    got = dict(out or {})
    wanted = {"dx": like, "df": f, "dgate": gate, "drscale": rscale, "dpost_weight": post_weight, "dpost_bias": post_bias,
              "dnext_weight": next_weight if dn is not None else None, "dnext_bias": next_bias if dn is not None else None}
    for name, t in wanted.items():
        if t is None:
            got[name] = None
        elif got.get(name) is None:
            got[name] = torch.empty_like(t)
    shape = like.shape

    def vec(t, name):
        return t if t is None else _ptr(t, torch.float32, (C,), name)

    def act(t, name):
        return t if t is None else _ptr(t, like.dtype, shape, name)

    _, dgp = _gate_kind(got["dgate"], like, "dgate")
    code = _dtype_code(like)
    if workspace is None:
        workspace = like.new_empty(max(nm_residual_norm_bwd_workspace_bytes(B, C, T, code), 256), dtype=torch.uint8)
        if stream is not None:
            workspace.record_stream(stream)  # (it is given back when this call returns)
    st = lib().nm_residual_norm_bwd(
        B, C, T, act(dy, "dy"), act(dn, "dn"), act(y, "y"), act(f, "f"), gp, kind, vec(rscale, "rscale"),
        vec(post_weight, "post_weight"), vec(post_bias, "post_bias"), vec(next_weight if dn is not None else None, "next_weight"), eps,
        _ptr(lengths, torch.int32, (B,), "lengths"), act(got["dx"], "dx"), act(got["df"], "df"), dgp, vec(got["drscale"], "drscale"),
        vec(got["dpost_weight"], "dpost_weight"), vec(got["dpost_bias"], "dpost_bias"), vec(got["dnext_weight"], "dnext_weight"),
        vec(got["dnext_bias"], "dnext_bias"), flags, code, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_residual_norm_bwd")
    return got


# ---- AdamW over many tensors (include/nm_adamw.h) -----------------------------------------------
class AdamWPlan:
    """The tensors of a step and their description on host and device.  Keeps the tensors alive."""

    def __init__(self, host, device, tensors, state_bits):
        self.host, self.device, self.tensors, self.state_bits = host, device, tensors, state_bits


def nm_adamw_plan(params, grads, m, v, *, m_scales=None, v_scales=None, copies=None, weight_decay=0.0) -> AdamWPlan:
    """Plan of a step over lists of device tensors of any shapes: float32 params and grads, m and v (float32, or uint8 E4M3 codes
    with the float32 scales of their blocks of 256: then states are held in 8 bits), copies (bfloat16 tensors or None each, or
    None).  weight_decay: a number or one per tensor."""
    torch = _torch()
    count = len(params)
    bits = 32 if m_scales is None else 8
    if (m_scales is None) != (v_scales is None):
        raise ValueError("m_scales and v_scales go together")
    none = [None] * count
    decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * count
    lists = {"params": params, "grads": grads, "m": m, "v": v, "m_scales": m_scales or none, "v_scales": v_scales or none,
             "copies": copies or none, "weight_decay": decay}
    for name, ts in lists.items():
        if len(ts) != count:
            raise ValueError(f"{name} must have {count} entries, got {len(ts)}")
    table = (AdamWTensor * max(count, 1))()
    state = torch.float32 if bits == 32 else torch.uint8
    for i in range(count):
        n = params[i].numel()

        def ptr(t, dtype, name, numel):
            if t is not None and t.numel() != numel:
                raise ValueError(f"{name}[{i}] must have {numel} elements, got {t.numel()}")
            return _ptr(t, dtype, None, f"{name}[{i}]")

        blocks = (n + 255) // 256
        table[i] = AdamWTensor(ptr(params[i], torch.float32, "params", n), ptr(grads[i], torch.float32, "grads", n),
                               ptr(m[i], state, "m", n), ptr(v[i], state, "v", n),
                               ptr(lists["m_scales"][i], torch.float32, "m_scales", blocks),
                               ptr(lists["v_scales"][i], torch.float32, "v_scales", blocks),
                               ptr(lists["copies"][i], torch.bfloat16, "copies", n), n, float(decay[i]))
    size = int(lib().nm_adamw_plan_bytes(table, count, bits))
    if not size:
        raise NmError(NM_ERR_BAD_ARG, "nm_adamw_plan_bytes")
    host = torch.empty(size, dtype=torch.uint8)
    st = lib().nm_adamw_plan(table, count, bits, host.data_ptr(), size)
    if st != NM_OK:
        raise NmError(st, "nm_adamw_plan")
    return AdamWPlan(host, host.to(params[0].device), lists, bits)


def nm_adamw_step(plan: AdamWPlan, *, lr, beta1=0.9, beta2=0.999, eps=1e-8, step, grad_scale=None, seed=0, stream=None) -> None:
    """One step over the tensors of the plan; step counts from 1.  grad_scale: float32 device tensor of one element that multiplies
    the gradients.  seed: of the rounding of 8-bit states, another one each step."""
    if grad_scale is not None and grad_scale.numel() != 1:
        raise ValueError(f"grad_scale must have one element, got {grad_scale.numel()}")
    st = lib().nm_adamw_step(plan.host.data_ptr(), plan.device.data_ptr(), plan.host.numel(), lr, beta1, beta2, eps, step,
                             _ptr(grad_scale, _torch().float32, None, "grad_scale"), seed & 0xFFFFFFFF, _stream(stream))
    if st != NM_OK:
        raise NmError(st, "nm_adamw_step")
