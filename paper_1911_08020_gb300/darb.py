"""Python binding of libdarb (include/darb.h): argument marshalling only.

Every function has the name of the C call it wraps and forwards torch tensors
as raw device pointers plus the current CUDA stream.  All arithmetic happens in
the library's CUDA kernels; if ``libdarb.so`` is missing or a call fails, a
``DarbError`` is raised -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading
from dataclasses import dataclass
from typing import NamedTuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdarb.so")

OK, ERR_INVALID_ARG, ERR_NONFINITE, ERR_OOM, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED = range(7)
F32, BF16 = 0, 1
PATH_AUTO, PATH_CUDA_CORES, PATH_TENSOR_CORES = 0, 1, 2
TOKEN_ROWS, TOKEN_COLUMNS = 0, 1
GATES_LOGITS, GATES_VALUES = 0, 1
PER_TOKEN, PER_SEQUENCE = 0, 1
MAX_BLOCK = 256
MAX_TOP = 32
ADAMW_BLOCK = 256

_lock = threading.Lock()
_lib = None


class DarbError(RuntimeError):
    def __init__(self, status: int, call: str):
        name = status_string(status) if _lib is not None else str(status)
        super().__init__(f"{call} failed: {name}")
        self.status = status


class _Info(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("nnzb", ctypes.c_int64),
                ("wtype", ctypes.c_int), ("nbins", ctypes.c_int32), ("ngroups", ctypes.c_int32),
                ("value_bytes", ctypes.c_int64), ("offset_bytes", ctypes.c_int64),
                ("meta_bytes", ctypes.c_int64), ("index_bits_min", ctypes.c_int64),
                ("device_bytes", ctypes.c_int64)]


def lib():
    """The loaded libdarb.so (raises if it has not been built)."""
    global _lib
    L = _lib
    if L is not None:
        return L
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise DarbError(ERR_CUDA, f"load {LIB_PATH} (not built; run __graft_entry__.build())")
            L = ctypes.CDLL(LIB_PATH)
            P, I64, I32, S = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
            sig = {
                "darb_assign_block_sizes": [P, I64, I64, I32, I32, P],
                "darb_assign_from_weights": [P, ctypes.c_int, I64, I64, I64, I64, I32, I32, P, P, S],
                "darb_encode": [P, ctypes.c_int, I64, I64, I64, P, P, S],
                "darb_reencode": [P, P, I64, S],
                "darb_reencode_host": [P, P, I64, P, S],
                "darb_sync_status": [P, S],
                "darb_spmm": [P, P, I64, I64, P, I64, S],
                "darb_spmm_ex": [P, P, I64, I64, P, I64, ctypes.c_int, S],
                "darb_spmm_host": [P, P, I64, I64, P, I64, P, P, S],
                "darb_spmm_path": [P, I64, P, P],
                "darb_lstm_step": [P, I64, I64, I64, P, P, P, P, P, P, S],
                "darb_lstm_step_noalloc": [P, I64, I64, I64, P, P, P, P, P, P, S],
                "darb_gru_step": [P, I64, I64, I64, P, P, P, P, P, S],
                "darb_lstm_sequence": [P, I64, I64, I64, I64, P, P, P, P, P, P, P, S],
                "darb_gru_sequence": [P, I64, I64, I64, I64, P, P, P, P, P, S],
                "darb_rnn_reserve": [P, I64],
                "darb_info": [P, P],
                "darb_export": [P, P, P, P, P],
                "darb_import": [P, P, P, ctypes.c_int, I64, I64, P, S],
                "darb_destroy": [P],
                "darb_set_pdl": [ctypes.c_int],
                "darb_token_logprobs": [P, ctypes.c_int, ctypes.c_int, I64, I64, I64, P, I32, P, P, P, P, P, S],
                "darb_token_logprobs_grad": [P, ctypes.c_int, ctypes.c_int, I64, I64, I64, P, P, P, P, P, P, I64, S],
                "darb_layer_norm": [P, ctypes.c_int, ctypes.c_int, I64, I64, I64, I64, P, P, ctypes.c_float, P, I64,
                                    P, P, S],
                "darb_layer_norm_grad": [P, I64, P, I64, ctypes.c_int, ctypes.c_int, I64, I64, I64, P, P, P, P, I64,
                                         P, P, P, S],
                "darb_layer_norm_grad_work": [ctypes.c_int, I64, I64, I64, P],
                "darb_gated_scan": [P, I64, I64, P, I64, I64, ctypes.c_int, ctypes.c_int, ctypes.c_int, I64, I64, I64, P, P,
                                    I64, I64, P, S],
                "darb_gated_scan_grad": [P, I64, I64, P, I64, I64, P, I64, I64, P, I64, I64, ctypes.c_int, ctypes.c_int,
                                         ctypes.c_int, I64, I64, I64, P, P, P, I64, I64, P, I64, I64, P, S],
                "darb_policy_loss": [I64, I64, P, P, P, P, P, P, P, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                     ctypes.c_double, ctypes.c_int, ctypes.c_int, P, P, P, P, S],
                "darb_policy_loss_work": [I64, P],
                "darb_adamw_create": [I32, P, P, P, P, P, P, P, ctypes.c_int, P, S],
                "darb_adamw_step": [P, P, P, I64, ctypes.c_uint64, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                    ctypes.c_double, ctypes.c_double, S],
                "darb_adamw_sync_status": [P, S],
                "darb_adamw_destroy": [P],
                "darb_muon_create": [I32, P, P, P, P, P, ctypes.c_int, P, S],
                "darb_muon_step": [P, P, P, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_int,
                                   S],
                "darb_muon_sync_status": [P, S],
                "darb_muon_destroy": [P],
            }
            for name, args in sig.items():
                fn = getattr(L, name)
                fn.argtypes = args
                fn.restype = ctypes.c_int
            L.darb_status_string.argtypes = [ctypes.c_int]
            L.darb_status_string.restype = ctypes.c_char_p
            _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().darb_status_string(int(status)).decode()


def _check(status: int, call: str):
    if status != OK:
        raise DarbError(status, call)


# The small calls of this module are bound by the host: a cell step runs 8 us on
# the device.  So what every call does is kept cheap: torch is looked up once,
# and the current stream's handle is read without building a Stream object
# (0.2 us against 3.0).
_torch = None
_raw_stream = None


def _load_torch():
    global _torch, _raw_stream
    import torch
    get, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))

    def raw():
        if get is None or device is None or not torch.cuda.is_initialized():
            return int(torch.cuda.current_stream().cuda_stream)
        return get(device())

    _raw_stream = raw
    _torch = torch
    return torch


def _ptr(t) -> int | None:
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        if _raw_stream is None:
            _load_torch()
        return _raw_stream()
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise DarbError(ERR_INVALID_ARG, f"dtype {t.dtype} (need float32 or bfloat16)")


def _require_cuda_f32(t, name):
    if t is None:
        return
    if not t.is_cuda or t.dtype != (_torch or _load_torch()).float32:
        raise DarbError(ERR_INVALID_ARG, f"{name} must be a CUDA float32 tensor")


@dataclass
class Handle:
    """An encoded DARB matrix living on the GPU (owned; free with darb_destroy)."""
    ptr: int
    rows: int
    cols: int
    wtype: int

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        darb_destroy(self)


def darb_assign_block_sizes(row_nnz, cols: int, m_min: int = 1, m_max: int = MAX_BLOCK) -> np.ndarray:
    nnz = np.ascontiguousarray(row_nnz, dtype=np.int64)
    out = np.zeros(nnz.shape[0], dtype=np.int32)
    _check(lib().darb_assign_block_sizes(nnz.ctypes.data, nnz.shape[0], int(cols), int(m_min),
                                         int(m_max), out.ctypes.data), "darb_assign_block_sizes")
    return out


def darb_assign_from_weights(W, keep: int, m_min: int = 1, m_max: int = MAX_BLOCK, stream=None,
                             ldw: int | None = None):
    """(row_nnz, m): each row's count of the `keep` weights of largest magnitude of
    the CUDA tensor W (rows x cols, float32 or bfloat16) and the block sizes they give."""
    code = _dtype_code(W)
    if W.dim() != 2 or not W.is_cuda or W.stride(1) != 1:
        raise DarbError(ERR_INVALID_ARG, "darb_assign_from_weights: W must be a 2-D CUDA tensor with unit column stride")
    rows, cols = W.shape
    ldw = W.stride(0) if ldw is None else ldw
    nnz = np.zeros(rows, dtype=np.int64)
    m = np.zeros(rows, dtype=np.int32)
    _check(lib().darb_assign_from_weights(_ptr(W), code, rows, cols, int(ldw), int(keep), int(m_min), int(m_max),
                                          nnz.ctypes.data, m.ctypes.data, _stream(stream)),
           "darb_assign_from_weights")
    return nnz, m


def darb_encode(W, m, stream=None, ldw: int | None = None) -> Handle:
    """Encode a CUDA tensor W (rows x cols, float32 or bfloat16) with block sizes m."""
    code = _dtype_code(W)
    if W.dim() != 2 or not W.is_cuda or W.stride(1) != 1:
        raise DarbError(ERR_INVALID_ARG, "darb_encode: W must be a 2-D CUDA tensor with unit column stride")
    rows, cols = W.shape
    ldw = W.stride(0) if ldw is None else ldw
    mm = np.ascontiguousarray(m, dtype=np.int32)
    if mm.shape != (rows,):
        raise DarbError(ERR_INVALID_ARG, "darb_encode: m must have one entry per row")
    out = ctypes.c_void_p()
    _check(lib().darb_encode(_ptr(W), code, rows, cols, ldw, mm.ctypes.data, ctypes.byref(out),
                             _stream(stream)), "darb_encode")
    return Handle(out.value, rows, cols, code)


def darb_reencode(h: Handle, W, stream=None):
    _check(lib().darb_reencode(h.ptr, _ptr(W), W.stride(0), _stream(stream)), "darb_reencode")


def darb_reencode_host(h: Handle, W, W_dev, stream=None):
    """darb_reencode from a host W (CPU tensor, rows x cols, row stride ldw) through
    the caller's device buffer W_dev (same shape and row stride)."""
    if W.is_cuda or not W_dev.is_cuda or W.dtype != W_dev.dtype:
        raise DarbError(ERR_INVALID_ARG, "darb_reencode_host: W on the host, W_dev on the device, one dtype")
    if W.shape != W_dev.shape or W.stride() != W_dev.stride() or W.stride(1) != 1:
        raise DarbError(ERR_INVALID_ARG, "darb_reencode_host: W and W_dev of one row-major layout")
    _check(lib().darb_reencode_host(h.ptr, _ptr(W), W.stride(0), _ptr(W_dev), _stream(stream)),
           "darb_reencode_host")


def darb_sync_status(h: Handle, stream=None):
    """Synchronise and raise if the handle's kernels recorded a NaN or a timeout."""
    _check(lib().darb_sync_status(h.ptr, _stream(stream)), "darb_sync_status")


def darb_spmm(h: Handle, X, Y=None, stream=None):
    """Y = W_darb X for X (cols x batch, CUDA float32); returns Y."""
    return darb_spmm_ex(h, X, Y, PATH_AUTO, stream)


def darb_spmm_ex(h: Handle, X, Y=None, path: int = PATH_AUTO, stream=None):
    """darb_spmm with the kernel family chosen (PATH_AUTO, PATH_CUDA_CORES, PATH_TENSOR_CORES)."""
    _require_cuda_f32(X, "X")
    if X.dim() == 1:
        X = X.view(-1, 1)
    shape, strides = X.shape, X.stride()
    batch = shape[1]
    if strides[1] != 1 and batch > 1:
        raise DarbError(ERR_INVALID_ARG, "darb_spmm: X must have a contiguous batch dimension")
    if Y is None:
        Y = _torch.empty((h.rows, batch), dtype=_torch.float32, device=X.device)
    else:
        _require_cuda_f32(Y, "Y")
    ldx = strides[0] if shape[0] > 1 else batch
    ldy = Y.stride(0) if Y.shape[0] > 1 else batch
    if path == PATH_AUTO:
        _check(lib().darb_spmm(h.ptr, X.data_ptr(), ldx, batch, Y.data_ptr(), ldy, _stream(stream)), "darb_spmm")
    else:
        _check(lib().darb_spmm_ex(h.ptr, X.data_ptr(), ldx, batch, Y.data_ptr(), ldy, int(path), _stream(stream)),
               "darb_spmm_ex")
    return Y


def darb_spmm_host(h: Handle, X, Y, X_dev, Y_dev, stream=None):
    """darb_spmm with X (cols x batch) and Y (rows x batch) host float32 tensors
    (rows strided, columns contiguous) through the caller's dense device buffers
    X_dev (cols x batch) and Y_dev (rows x batch); returns Y."""
    import torch
    for t, n, cuda in ((X, "X", False), (Y, "Y", False), (X_dev, "X_dev", True), (Y_dev, "Y_dev", True)):
        if t.dtype != torch.float32 or t.is_cuda != cuda or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
            raise DarbError(ERR_INVALID_ARG, f"darb_spmm_host: {n} must be a 2-D float32 "
                                             f"{'CUDA' if cuda else 'host'} tensor with contiguous columns")
    batch = X.shape[1]
    if (X_dev.shape != X.shape or Y.shape != (h.rows, batch) or Y_dev.shape != Y.shape or
            not X_dev.is_contiguous() or not Y_dev.is_contiguous()):
        raise DarbError(ERR_INVALID_ARG, "darb_spmm_host: shapes, or device buffers not dense")
    ldx = X.stride(0) if X.shape[0] > 1 else batch
    ldy = Y.stride(0) if Y.shape[0] > 1 else batch
    _check(lib().darb_spmm_host(h.ptr, _ptr(X), ldx, batch, _ptr(Y), ldy, _ptr(X_dev), _ptr(Y_dev),
                                _stream(stream)), "darb_spmm_host")
    return Y


def darb_spmm_path(h: Handle, batch: int) -> tuple[int, int]:
    """(path, kernels): the kernel family darb_spmm takes for this batch and its launches per call."""
    path, kernels = ctypes.c_int(), ctypes.c_int32()
    _check(lib().darb_spmm_path(h.ptr, int(batch), ctypes.byref(path), ctypes.byref(kernels)), "darb_spmm_path")
    return path.value, kernels.value


def darb_lstm_step(h: Handle, I: int, H: int, B: int, x, h_prev, c_prev, bias, h_out, c_out,
                   stream=None):
    for t, n in ((x, "x"), (h_prev, "h_prev"), (c_prev, "c_prev"), (bias, "bias"),
                 (h_out, "h_out"), (c_out, "c_out")):
        _require_cuda_f32(t, n)
    _check(lib().darb_lstm_step(h.ptr, I, H, B, _ptr(x), _ptr(h_prev), _ptr(c_prev), _ptr(bias),
                                _ptr(h_out), _ptr(c_out), _stream(stream)), "darb_lstm_step")


def darb_lstm_step_noalloc(h: Handle, I: int, H: int, B: int, x, h_prev, c_prev, bias, h_out, c_out,
                           stream=None):
    """darb_lstm_step with its scratch in the library's fixed 4 MiB array: no
    allocation at call time (for callers that cannot let a library allocate)."""
    for t, n in ((x, "x"), (h_prev, "h_prev"), (c_prev, "c_prev"), (bias, "bias"),
                 (h_out, "h_out"), (c_out, "c_out")):
        _require_cuda_f32(t, n)
    _check(lib().darb_lstm_step_noalloc(h.ptr, I, H, B, _ptr(x), _ptr(h_prev), _ptr(c_prev),
                                        _ptr(bias), _ptr(h_out), _ptr(c_out), _stream(stream)),
           "darb_lstm_step_noalloc")


def darb_gru_step(h: Handle, I: int, H: int, B: int, x, h_prev, b_ih, b_hh, h_out, stream=None):
    for t, n in ((x, "x"), (h_prev, "h_prev"), (b_ih, "b_ih"), (b_hh, "b_hh"), (h_out, "h_out")):
        _require_cuda_f32(t, n)
    _check(lib().darb_gru_step(h.ptr, I, H, B, _ptr(x), _ptr(h_prev), _ptr(b_ih), _ptr(b_hh),
                               _ptr(h_out), _stream(stream)), "darb_gru_step")


def darb_lstm_sequence(h: Handle, T: int, I: int, H: int, B: int, x_seq, h0, c0, bias, h_seq,
                       c_seq=None, c_last=None, stream=None):
    """T LSTM steps in one persistent launch: x_seq (T, I, B) -> h_seq (T, H, B),
    optionally every c_t (c_seq) and the last c (c_last)."""
    for t, n in ((x_seq, "x_seq"), (h0, "h0"), (c0, "c0"), (bias, "bias"), (h_seq, "h_seq"),
                 (c_seq, "c_seq"), (c_last, "c_last")):
        _require_cuda_f32(t, n)
    _check(lib().darb_lstm_sequence(h.ptr, T, I, H, B, _ptr(x_seq), _ptr(h0), _ptr(c0), _ptr(bias),
                                    _ptr(h_seq), _ptr(c_seq), _ptr(c_last), _stream(stream)),
           "darb_lstm_sequence")


def darb_gru_sequence(h: Handle, T: int, I: int, H: int, B: int, x_seq, h0, b_ih, b_hh, h_seq, stream=None):
    """T GRU steps in one persistent launch: x_seq (T, I, B) -> h_seq (T, H, B)."""
    for t, n in ((x_seq, "x_seq"), (h0, "h0"), (b_ih, "b_ih"), (b_hh, "b_hh"), (h_seq, "h_seq")):
        _require_cuda_f32(t, n)
    _check(lib().darb_gru_sequence(h.ptr, T, I, H, B, _ptr(x_seq), _ptr(h0), _ptr(b_ih), _ptr(b_hh),
                                   _ptr(h_seq), _stream(stream)), "darb_gru_sequence")


def darb_rnn_reserve(h: Handle, max_batch: int):
    _check(lib().darb_rnn_reserve(h.ptr, int(max_batch)), "darb_rnn_reserve")


def darb_info(h: Handle) -> dict:
    info = _Info()
    _check(lib().darb_info(h.ptr, ctypes.byref(info)), "darb_info")
    return {name: getattr(info, name) for name, _ in _Info._fields_}


def darb_export(h: Handle):
    """(val, off, blk_ptr, m) in canonical (row, j) block order; val is float32 or uint16 bf16 bits."""
    info = darb_info(h)
    nnzb = info["nnzb"]
    val = np.zeros(nnzb, dtype=np.uint16 if h.wtype == BF16 else np.float32)
    off = np.zeros(nnzb, dtype=np.uint8)
    bp = np.zeros(h.rows + 1, dtype=np.int64)
    m = np.zeros(h.rows, dtype=np.int32)
    _check(lib().darb_export(h.ptr, val.ctypes.data, off.ctypes.data, bp.ctypes.data, m.ctypes.data),
           "darb_export")
    return val, off, bp, m


def darb_import(val, off, m, wtype: int, rows: int, cols: int, stream=None) -> Handle:
    v = np.ascontiguousarray(val, dtype=np.uint16 if wtype == BF16 else np.float32)
    o = np.ascontiguousarray(off, dtype=np.uint8)
    mm = np.ascontiguousarray(m, dtype=np.int32)
    out = ctypes.c_void_p()
    _check(lib().darb_import(v.ctypes.data, o.ctypes.data, mm.ctypes.data, int(wtype), int(rows),
                             int(cols), ctypes.byref(out), _stream(stream)), "darb_import")
    return Handle(out.value, rows, cols, wtype)


def darb_destroy(h: Handle | None):
    if h is None or h.ptr is None:
        return
    _check(lib().darb_destroy(h.ptr), "darb_destroy")
    h.ptr = None


def darb_set_pdl(enabled: bool):
    """Launch the library's kernels with (default) or without programmatic dependent launch."""
    _check(lib().darb_set_pdl(1 if enabled else 0), "darb_set_pdl")


# ---- scoring and training around a pruned layer ----

def _refuse(call: str, what: str):
    raise DarbError(ERR_INVALID_ARG, f"{call}: {what}")


def _value_code(t, call: str, name: str) -> int:
    """The type code of a CUDA tensor of activations."""
    torch = _torch or _load_torch()
    if not t.is_cuda:
        _refuse(call, f"{name} must be a CUDA tensor")
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    _refuse(call, f"{name} must be float32 or bfloat16")


def _vector(t, n: int, dtype, call: str, name: str) -> int | None:
    """The pointer of a dense CUDA vector of n values, or None."""
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        _refuse(call, f"{name} must be a contiguous CUDA {dtype} tensor of {n} values")
    return t.data_ptr()


def _new(shape, dtype, device, stream):
    """A new tensor, kept from reuse while `stream` (if it is not the current one) may still work on it."""
    t = _torch.empty(shape, dtype=dtype, device=device)
    if stream is not None:
        t.record_stream(_torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream)
    return t


def _zero(t, stream):
    """Zeros in a new tensor, in the order of `stream`."""
    if stream is None:
        t.zero_()
        return
    with _torch.cuda.stream(_torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        t.zero_()


def _tokens(t, dim: int, call: str, name: str) -> tuple[int, int, int, int, int]:
    """(layout, steps, tokens, features, ld) of a tensor whose features lie along `dim`: 2-D with
    either axis contiguous, or 3-D (steps, features, tokens) with contiguous tokens."""
    shape, strides = t.shape, t.stride()
    if len(shape) == 2:
        if dim not in (-2, -1, 0, 1):
            _refuse(call, f"no axis {dim}")
        f, n = (shape[1], shape[0]) if dim % 2 else shape
        fs, ns = (strides[1], strides[0]) if dim % 2 else strides
        if fs == 1 or f == 1:
            return TOKEN_ROWS, 1, n, f, ns if n > 1 else f
        if ns == 1 or n == 1:
            return TOKEN_COLUMNS, 1, n, f, fs
        _refuse(call, f"an axis of {name} must be contiguous")
    if len(shape) != 3 or dim not in (1, -2):
        _refuse(call, f"{name} must be 2-D, or 3-D (steps, features, tokens) with dim=1")
    steps, f, n = shape
    ld = strides[1] if f > 1 else strides[0] if steps > 1 else n
    if (n > 1 and strides[2] != 1) or (steps > 1 and strides[0] != f * ld):
        _refuse(call, f"{name} must have contiguous tokens and steps one after the other")
    return TOKEN_COLUMNS, steps, n, f, ld


def _single_token(layout: int, n: int, f: int, ld: int, x, others, dim: int) -> tuple[int, int]:
    """(layout, ld) of one token's features x, which can be taken as a row if they are contiguous, but have
    to be taken as a column where those of another tensor of the call are not."""
    if n == 1 and layout == TOKEN_ROWS and x.dim() == 2:
        if any(t is not None and t.dim() == 2 and t.stride()[dim] != 1 for t in others):
            return TOKEN_COLUMNS, x.stride()[dim] if f > 1 else 1
    return layout, ld


def _same_tokens(t, like, ld: int, dim: int, layout: int, call: str, name: str) -> int:
    """The leading dimension of a tensor of the shape, type and layout of another, whose own is `ld`."""
    if not t.is_cuda or t.dtype != like.dtype or t.shape != like.shape:
        _refuse(call, f"{name} must be a CUDA tensor of the input's shape and type")
    strides = t.stride()
    if strides == like.stride():
        return ld
    f, n = (t.shape[dim], t.shape[1 - dim % 2 if t.dim() == 2 else 2])
    fs, ns = (strides[dim], strides[1 - dim % 2 if t.dim() == 2 else 2])
    steps = 1 if t.dim() == 2 else t.shape[0]
    if layout == TOKEN_ROWS:
        if f > 1 and fs != 1:
            _refuse(call, f"{name} must have contiguous features, as the input")
        return ns if n > 1 else f
    ld = fs if f > 1 else strides[0] if steps > 1 else n
    if (n > 1 and ns != 1) or (steps > 1 and strides[0] != f * ld):
        _refuse(call, f"{name} must have contiguous tokens, as the input")
    return ld


class TokenLogprobs(NamedTuple):
    """Results of darb_token_logprobs: float32 (tokens,) and, of the k alternatives, float32 and int32 (tokens, k)."""
    logprob: object
    entropy: object
    lse: object
    top_logprob: object
    top_index: object

    @staticmethod
    def empty(tokens: int, k: int = 0, device="cuda", stream=None) -> "TokenLogprobs":
        """Buffers for the results of `tokens` tokens, to be passed as `out`."""
        torch = _torch or _load_torch()
        f32 = [_new((tokens,), torch.float32, device, stream) for _ in range(3)]
        return TokenLogprobs(*f32, _new((tokens, k), torch.float32, device, stream),
                             _new((tokens, k), torch.int32, device, stream))


def darb_token_logprobs(logits, targets=None, k: int = 0, dim: int = -1, out: TokenLogprobs | None = None,
                        stream=None) -> TokenLogprobs:
    """Log probability of the given entries, entropy, log of the sum of exponentials and the k most
    probable entries of each token, from its logits.

    logits: 2-D float32 or bfloat16, the vocabulary along `dim` (-1: tokens x vocab; 0: vocab x tokens,
    what darb_spmm returns), either axis contiguous.  targets: int64 (tokens,), negative for none; without
    targets there is no logprob.  out: buffers to write (entries may be None: not wanted).  What the call does
    not compute is None in what it returns, also where `out` has a buffer for it."""
    call = "darb_token_logprobs"
    code = _value_code(logits, call, "logits")
    if logits.dim() != 2:
        _refuse(call, "logits must be 2-D")
    if k < 0:
        _refuse(call, "k must not be negative")
    layout, _, n, v, ld = _tokens(logits, dim, call, "logits")
    torch = _torch
    if out is None:
        out = TokenLogprobs.empty(n, k, logits.device, stream)
    elif k == 0 and any(t is not None and t.numel() for t in out[3:]):
        out = out._replace(top_logprob=None, top_index=None)
    if targets is None:
        out = out._replace(logprob=None)
    f32 = torch.float32
    logprob = None if targets is None else _vector(out.logprob, n, f32, call, "logprob")
    top = (_vector(out.top_logprob, n * k, f32, call, "top_logprob"),
           _vector(out.top_index, n * k, torch.int32, call, "top_index")) if k else (None, None)
    _check(lib().darb_token_logprobs(logits.data_ptr(), code, layout, n, v, ld,
                                     None if logprob is None else _vector(targets, n, torch.int64, call, "targets"), k, logprob,
                                     _vector(out.entropy, n, f32, call, "entropy"), _vector(out.lse, n, f32, call, "lse"),
                                     *top, _stream(stream)), call)
    return out


def darb_token_logprobs_grad(logits, targets, lse, d_logprob, entropy=None, d_entropy=None, dim: int = -1, out=None,
                             stream=None):
    """The gradient with respect to the logits, given those of log probability (d_logprob) and entropy
    (d_entropy); lse and entropy are the forward call's.  out: a tensor of the logits' shape, type and
    layout, or the logits themselves; a new one if None."""
    call = "darb_token_logprobs_grad"
    code = _value_code(logits, call, "logits")
    if logits.dim() != 2:
        _refuse(call, "logits must be 2-D")
    layout, _, n, v, ld = _tokens(logits, dim, call, "logits")
    torch = _torch
    if out is None:
        out = _new((n, v) if layout == TOKEN_ROWS else (v, n), logits.dtype, logits.device, stream)
        if (layout == TOKEN_ROWS) != (dim % 2 == 1):
            out = out.t()
    layout, ld = _single_token(layout, n, v, ld, logits, (out,), dim)
    ld_out = _same_tokens(out, logits, ld, dim, layout, call, "out")
    f32 = torch.float32
    _check(lib().darb_token_logprobs_grad(logits.data_ptr(), code, layout, n, v, ld,
                                          _vector(targets, n, torch.int64, call, "targets"), _vector(lse, n, f32, call, "lse"),
                                          _vector(entropy, n, f32, call, "entropy"),
                                          _vector(d_logprob, n, f32, call, "d_logprob"),
                                          _vector(d_entropy, n, f32, call, "d_entropy"), out.data_ptr(), ld_out,
                                          _stream(stream)), call)
    return out


def darb_layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, dim: int = -1, y=None, mean=None, rstd=None,
                    stream=None):
    """(y, mean, rstd): layer norm over the features of each token, which lie along `dim`.

    x: float32 or bfloat16, 2-D with either axis contiguous (dim=-1: tokens x features; dim=0: features x
    tokens, as the steps write h) or 3-D (steps, features, tokens) with dim=1, as the sequence calls write
    h_seq.  gamma, beta: float32 (features,) or None.  y may be x; mean and rstd: float32, a value a token."""
    call = "darb_layer_norm"
    code = _value_code(x, call, "x")
    layout, steps, n, f, ld = _tokens(x, dim, call, "x")
    f32 = _torch.float32
    if y is None:
        y = _new_like(x, dim, layout, steps, n, f, stream)
    layout, ld = _single_token(layout, n, f, ld, x, (y,), dim)
    lead = (steps, n) if x.dim() == 3 else (n,)
    if mean is None:
        mean = _new(lead, f32, x.device, stream)
    if rstd is None:
        rstd = _new(lead, f32, x.device, stream)
    _check(lib().darb_layer_norm(x.data_ptr(), code, layout, steps, n, f, ld, _vector(gamma, f, f32, call, "gamma"),
                                 _vector(beta, f, f32, call, "beta"), eps, y.data_ptr(),
                                 _same_tokens(y, x, ld, dim, layout, call, "y"), _vector(mean, steps * n, f32, call, "mean"),
                                 _vector(rstd, steps * n, f32, call, "rstd"), _stream(stream)), call)
    return y, mean, rstd


def _new_like(x, dim: int, layout: int, steps: int, n: int, f: int, stream):
    """A dense tensor of x's shape and type whose contiguous axis is x's."""
    if x.dim() == 3:
        return _new((steps, f, n), x.dtype, x.device, stream)
    t = _new((n, f) if layout == TOKEN_ROWS else (f, n), x.dtype, x.device, stream)
    return t if (layout == TOKEN_ROWS) == (dim % 2 == 1) else t.t()


def darb_layer_norm_grad(dy, x, gamma, mean, rstd, dim: int = -1, dx=None, dgamma=None, dbeta=None, weights: bool = True,
                         work=None, stream=None):
    """(dx, dgamma, dbeta): the backward pass of darb_layer_norm (dx may be dy).  weights=False leaves
    dgamma and dbeta out (None).  work: scratch of darb_layer_norm_grad_work bytes; from the
    device's memory pool if None."""
    call = "darb_layer_norm_grad"
    code = _value_code(x, call, "x")
    layout, steps, n, f, ld = _tokens(x, dim, call, "x")
    f32 = _torch.float32
    if dx is None:
        dx = _new_like(x, dim, layout, steps, n, f, stream)
    layout, ld = _single_token(layout, n, f, ld, x, (dy, dx), dim)
    pg = pb = pw = None
    if weights:
        if dgamma is None:
            dgamma = _new((f,), f32, x.device, stream)
        if dbeta is None:
            dbeta = _new((f,), f32, x.device, stream)
        pg, pb = _vector(dgamma, f, f32, call, "dgamma"), _vector(dbeta, f, f32, call, "dbeta")
        if work is not None:
            need = darb_layer_norm_grad_work(layout, steps, n, f)
            if not work.is_cuda or not work.is_contiguous() or work.numel() * work.element_size() < need:
                _refuse(call, f"work must be a contiguous CUDA tensor of {need} bytes")
            pw = work.data_ptr()
    else:
        dgamma = dbeta = None
    _check(lib().darb_layer_norm_grad(dy.data_ptr(), _same_tokens(dy, x, ld, dim, layout, call, "dy"), x.data_ptr(), ld, code,
                                      layout, steps, n, f, _vector(gamma, f, f32, call, "gamma"),
                                      _vector(mean, steps * n, f32, call, "mean"), _vector(rstd, steps * n, f32, call, "rstd"),
                                      dx.data_ptr(), _same_tokens(dx, x, ld, dim, layout, call, "dx"), pg, pb, pw,
                                      _stream(stream)), call)
    return dx, dgamma, dbeta


def darb_layer_norm_grad_work(layout: int, steps: int, tokens: int, features: int) -> int:
    """Bytes of scratch that darb_layer_norm_grad needs (layout: TOKEN_ROWS or TOKEN_COLUMNS)."""
    need = ctypes.c_int64()
    _check(lib().darb_layer_norm_grad_work(layout, steps, tokens, features, ctypes.byref(need)),
           "darb_layer_norm_grad_work")
    return need.value


# ---- a gated linear recurrence ----

def _channel_axes(shape, strides, dim: int, call: str) -> tuple[int, int, int, int, int]:
    """(outer, steps, inner, outer axis, step axis) of tensors of one shape and these strides whose steps lie along
    `dim`: their other axes are one run of contiguous channels where that holds for all of them, else a strided
    axis and a contiguous one.  The outer axis is -1 where there is none."""
    nd = len(shape)
    if nd not in (2, 3) or not -nd <= dim < nd:
        _refuse(call, "x must be 2-D or 3-D, with its steps along dim")
    if dim < 0:
        dim += nd
    if nd == 2:
        axis = 1 - dim
        channels = shape[axis]
    else:
        a, axis = ((1, 2), (0, 2), (0, 1))[dim]
        na, nb = shape[a], shape[axis]
        channels = na * nb
        if nb == 1:
            axis = a
        elif na > 1 and channels:
            for s in strides:
                if s[a] != nb * s[axis]:
                    if any(t[axis] != 1 for t in strides):
                        _refuse(call, "the last axis of the channels must be contiguous, or all channels equally far apart")
                    return na, shape[dim], nb, a, dim
    if channels > 1:
        for s in strides:
            if s[axis] != 1:
                return channels, shape[dim], 1, axis, dim
    return 1, shape[dim], channels, -1, dim


def _scan_operand(t, dtype, s, outer: int, step: int, call: str, name: str):
    """(pointer, leading dimension, step) of a tensor with strides s, checked to be of x's type."""
    if t.dtype is not dtype or not t.is_cuda:
        _refuse(call, f"{name} must be a CUDA tensor of x's type")
    return t.data_ptr(), s[outer] if outer >= 0 else 0, s[step]


def _state_shape(x, dim: int):
    shape = list(x.shape)
    del shape[dim]
    return shape


def darb_gated_scan(gate, x, h0=None, dim: int = 0, gates: int = GATES_LOGITS, coupled: bool = True, h=None, h_last=None,
                    stream=None):
    """(h, h_last): the recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t over the steps along `dim`, every channel for
    itself, with a_t = sigmoid(gate_t) (GATES_VALUES: gate_t); coupled=False: without the factor 1 - a_t.

    gate, x: float32 or bfloat16, 2-D or 3-D, e.g. (steps, features, batch) with dim=0, as the sequence calls
    write; a product of all steps, viewed as (features, steps, batch), with dim=1; token rows (batch, steps,
    features) with dim=1.  Slices of wider tensors are taken as they are.  h0: float32 of x's shape without
    `dim`, the state before the first step (None: 0).  h: as x, and may be x; h_last: as h0, and may be h0."""
    call = "darb_gated_scan"
    code = _value_code(x, call, "x")
    f32, shape = _torch.float32, x.shape
    if h is None:
        h = _new(shape, x.dtype, x.device, stream)
    if gate.shape != shape or h.shape != shape:
        _refuse(call, "gate and h must have x's shape")
    gs, xs, hs = gate.stride(), x.stride(), h.stride()
    outer, steps, inner, oa, sa = _channel_axes(shape, (xs,) if gs == xs == hs else (gs, xs, hs), dim, call)
    if h_last is None:
        h_last = _new(_state_shape(x, sa), f32, x.device, stream)
    n, dtype = outer * inner, x.dtype
    _check(lib().darb_gated_scan(*_scan_operand(gate, dtype, gs, oa, sa, call, "gate"), x.data_ptr(), xs[oa] if oa >= 0 else 0, xs[sa],
                                 code, gates, bool(coupled), outer, steps, inner, _vector(h0, n, f32, call, "h0"),
                                 *_scan_operand(h, dtype, hs, oa, sa, call, "h"), _vector(h_last, n, f32, call, "h_last"),
                                 _stream(stream)), call)
    return h, h_last


def darb_gated_scan_grad(dh, gate, x, h, h0=None, d_last=None, dim: int = 0, gates: int = GATES_LOGITS, coupled: bool = True,
                         d_gate=None, d_x=None, d_h0=None, stream=None):
    """(d_gate, d_x, d_h0): the backward pass of darb_gated_scan, given the gradients of h (dh) and of h_last
    (d_last; None: 0).  h: the forward call's.  d_gate may be gate, d_x may be x, d_h0 may be d_last.  Without
    h0 there is no d_h0 (None) unless a buffer for it is given."""
    call = "darb_gated_scan_grad"
    code = _value_code(x, call, "x")
    f32, shape = _torch.float32, x.shape
    if d_gate is None:
        d_gate = _new(shape, x.dtype, x.device, stream)
    if d_x is None:
        d_x = _new(shape, x.dtype, x.device, stream)
    tensors = (dh, gate, x, h, d_gate, d_x)
    for t in tensors:
        if t is not x and t.shape != shape:
            _refuse(call, "dh, gate, h, d_gate and d_x must have x's shape")
    strides = [t.stride() for t in tensors]
    xs = strides[2]
    outer, steps, inner, oa, sa = _channel_axes(shape, (xs,) if strides.count(xs) == 6 else strides, dim, call)
    if d_h0 is None and h0 is not None:
        d_h0 = _new(_state_shape(x, sa), f32, x.device, stream)
    n, dtype, at = outer * inner, x.dtype, []
    for t, s, name in zip(tensors, strides, ("dh", "gate", "x", "h", "d_gate", "d_x")):
        if t.dtype is not dtype or not t.is_cuda:
            _refuse(call, f"{name} must be a CUDA tensor of x's type")
        at += (t.data_ptr(), s[oa] if oa >= 0 else 0, s[sa])
    _check(lib().darb_gated_scan_grad(*at[:12], code, gates, bool(coupled), outer, steps, inner,
                                      _vector(h0, n, f32, call, "h0"), _vector(d_last, n, f32, call, "d_last"), *at[12:],
                                      _vector(d_h0, n, f32, call, "d_h0"), _stream(stream)), call)
    return d_gate, d_x, d_h0


# ---- the loss of drawn answers ----

class PolicyLoss(NamedTuple):
    """Results of darb_policy_loss: stats, float32 (5,): loss, policy, kl, entropy, share of the clipped weight; the
    gradients of the loss, float32 (tokens,); and the call's scratch."""
    stats: object
    d_logprob: object
    d_entropy: object
    work: object

    @staticmethod
    def empty(tokens: int, device="cuda", entropy: bool = False, stream=None) -> "PolicyLoss":
        """Buffers for `tokens` tokens, to be passed as `out`."""
        torch = _torch or _load_torch()
        need = darb_policy_loss_work(tokens)
        return PolicyLoss(_new((5,), torch.float32, device, stream), _new((tokens,), torch.float32, device, stream),
                          _new((tokens,), torch.float32, device, stream) if entropy else None,
                          _new((need,), torch.uint8, device, stream) if need else None)


def darb_policy_loss(logprob, old_logprob, advantage, offsets, ref_logprob=None, entropy=None, mask=None, clip_low: float = 0.2,
                     clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, ratio: int = PER_TOKEN,
                     mean: int = PER_TOKEN, out: PolicyLoss | None = None, stream=None) -> PolicyLoss:
    """The clipped policy loss of answers that a model drew, with a KL term and an entropy bonus, and its
    gradients with respect to log probabilities and entropies, as darb_token_logprobs_grad takes them.

    logprob, old_logprob, ref_logprob, entropy: float32 (tokens,), the answers one after the other; advantage:
    float32 (sequences,); offsets: int64 (sequences + 1,), where each starts; mask: bool or uint8 (tokens,),
    the tokens that count.  ratio, mean: PER_TOKEN or PER_SEQUENCE.  out: buffers to write; new ones, with the
    gradients 0 outside of all sequences, if None."""
    call = "darb_policy_loss"
    torch = _torch or _load_torch()
    f32 = torch.float32
    n, sequences = logprob.numel(), advantage.numel()
    if out is None:
        out = PolicyLoss.empty(n, logprob.device, entropy is not None, stream)
        for t in out[1:3]:
            if t is not None:
                _zero(t, stream)
    if mask is not None and mask.dtype not in (torch.bool, torch.uint8):
        _refuse(call, "mask must be bool or uint8")
    work = out.work
    if work is not None:
        if n <= 4096:
            work = None
        else:
            need = darb_policy_loss_work(n)
            if not work.is_cuda or not work.is_contiguous() or work.numel() * work.element_size() < need:
                _refuse(call, f"work must be a contiguous CUDA tensor of {need} bytes")
    if out.stats is None or (n and out.d_logprob is None):
        _refuse(call, "stats and d_logprob must be there")
    _check(lib().darb_policy_loss(n, sequences, _vector(logprob, n, f32, call, "logprob"),
                                  _vector(old_logprob, n, f32, call, "old_logprob"),
                                  _vector(ref_logprob, n, f32, call, "ref_logprob"), _vector(entropy, n, f32, call, "entropy"),
                                  None if mask is None else _vector(mask, n, mask.dtype, call, "mask"),
                                  _vector(advantage, sequences, f32, call, "advantage"),
                                  _vector(offsets, sequences + 1, torch.int64, call, "offsets"), clip_low, clip_high, kl_coef,
                                  entropy_coef, ratio, mean, _vector(out.stats, 5, f32, call, "stats"),
                                  _vector(out.d_logprob, n, f32, call, "d_logprob"),
                                  _vector(out.d_entropy, n, f32, call, "d_entropy"),
                                  None if work is None else work.data_ptr(), _stream(stream)), call)
    return out


@functools.lru_cache(maxsize=64)
def darb_policy_loss_work(tokens: int) -> int:
    """Bytes of scratch that darb_policy_loss needs for so many tokens."""
    need = ctypes.c_int64()
    _check(lib().darb_policy_loss_work(tokens, ctypes.byref(need)), "darb_policy_loss_work")
    return need.value


class AdamW:
    """A plan of darb_adamw_create (owned; free with darb_adamw_destroy).  Holds on to its tensors."""

    def __init__(self, ptr: int, tensors, numels, grad_dtype):
        self.ptr, self.tensors, self.numels, self.grad_dtype = ptr, tensors, numels, grad_dtype
        self.pointers = (ctypes.c_void_p * len(numels))()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        darb_adamw_destroy(self)


def darb_adamw_create(params, m, v, m_scale=None, v_scale=None, copies=None, grad_dtype=None, stream=None) -> AdamW:
    """A plan for AdamW steps over the float32 CUDA tensors `params`, all tensors contiguous.

    m, v: the moments, float32 of the parameters' sizes; or, with m_scale and v_scale (float32, one value
    for every ADAMW_BLOCK elements of a tensor), float8_e4m3fn (or uint8) codes of m and of sqrt(v).
    copies: bfloat16 tensors (or None) that receive the rounded parameters, e.g. for darb_reencode.
    grad_dtype: float32 (default) or bfloat16."""
    call = "darb_adamw_create"
    torch = _torch or _load_torch()
    params, m, v = list(params), list(m), list(v)
    n = len(params)
    lists = [params, m, v] + [None if t is None else list(t) for t in (m_scale, v_scale, copies)]
    if any(t is not None and len(t) != n for t in lists):
        _refuse(call, "one state (and scale and copy) for every parameter")
    if (m_scale is None) != (v_scale is None):
        _refuse(call, "m_scale and v_scale go together")
    codes = (torch.float8_e4m3fn, torch.uint8)
    states = codes if m_scale is not None else (torch.float32,)
    grad_dtype = torch.float32 if grad_dtype is None else grad_dtype
    if grad_dtype not in (torch.float32, torch.bfloat16):
        _refuse(call, "grad_dtype must be float32 or bfloat16")
    kinds = [(torch.float32,), states, states, (torch.float32,), (torch.float32,), (torch.bfloat16,)]
    names = ("params", "m", "v", "m_scale", "v_scale", "copies")
    numels = [p.numel() for p in params]
    pointers = []
    for name, tensors, dtypes in zip(names, lists, kinds):
        if tensors is None:
            pointers.append(None)
            continue
        for t, size in zip(tensors, numels):
            if t is None and name == "copies":
                continue
            want = -(-size // ADAMW_BLOCK) if name.endswith("scale") else size
            if not t.is_cuda or t.dtype not in dtypes or t.numel() != want or not t.is_contiguous():
                _refuse(call, f"{name} must be contiguous CUDA tensors of {' or '.join(map(str, dtypes))}, {want} values here")
        pointers.append((ctypes.c_void_p * n)(*[None if t is None else t.data_ptr() for t in tensors]))
    out = ctypes.c_void_p()
    _check(lib().darb_adamw_create(n, (ctypes.c_int64 * n)(*numels), *pointers, BF16 if grad_dtype == torch.bfloat16 else F32,
                                   ctypes.byref(out), _stream(stream)), call)
    return AdamW(out.value, lists, numels, grad_dtype)


def _gradient_pointers(plan, grads, call: str):
    """The gradients of a plan's tensors (None where there is none) as an array of pointers."""
    pointers, dtype = plan.pointers, plan.grad_dtype
    if len(grads) != len(plan.numels):
        _refuse(call, "one gradient for every parameter")
    for i, (g, n) in enumerate(zip(grads, plan.numels)):
        if g is None:
            pointers[i] = None
            continue
        if g.dtype != dtype or not g.is_cuda or g.numel() != n or not g.is_contiguous():
            _refuse(call, f"gradient {i} must be a contiguous CUDA {dtype} tensor of {n} values")
        pointers[i] = g.data_ptr()
    return pointers


def darb_adamw_step(plan: AdamW, grads, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                    weight_decay: float = 0.01, grad_scale=None, seed: int | None = None, stream=None):
    """One step (step >= 1) with the gradients `grads` of the plan's tensors (None: that tensor is left as it
    is).  grad_scale: float32 CUDA scalar that multiplies every gradient.  seed: of the rounding of states in
    8 bits, the step itself if None."""
    call = "darb_adamw_step"
    pointers = _gradient_pointers(plan, grads, call)
    _check(lib().darb_adamw_step(plan.ptr, pointers, _vector(grad_scale, 1, (_torch or _load_torch()).float32, call, "grad_scale"),
                                 step, (step if seed is None else seed) & 0xFFFFFFFFFFFFFFFF, lr, beta1, beta2, eps,
                                 weight_decay, _stream(stream)), call)


def darb_adamw_sync_status(plan: AdamW, stream=None):
    """Synchronise and raise if a step's bounded wait gave up."""
    _check(lib().darb_adamw_sync_status(plan.ptr, _stream(stream)), "darb_adamw_sync_status")


def darb_adamw_destroy(plan: AdamW | None):
    if plan is None or plan.ptr is None:
        return
    _check(lib().darb_adamw_destroy(plan.ptr), "darb_adamw_destroy")
    plan.ptr = None


class Muon:
    """A plan of darb_muon_create (owned; free with darb_muon_destroy).  Holds on to its tensors."""

    def __init__(self, ptr: int, tensors, shapes, grad_dtype):
        self.ptr, self.tensors, self.shapes, self.grad_dtype = ptr, tensors, shapes, grad_dtype
        self.numels = [s.numel() for s in shapes]
        self.pointers = (ctypes.c_void_p * len(shapes))()

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        darb_muon_destroy(self)


def darb_muon_create(params, m, copies=None, grad_dtype=None, stream=None) -> Muon:
    """A plan for updates with orthogonalised momentum of the float32 CUDA matrices `params`, all contiguous.

    m: the momentum, float32 of the parameters' shapes.  copies: bfloat16 tensors (or None) that receive the
    rounded parameters, e.g. for darb_reencode.  grad_dtype: float32 (default) or bfloat16."""
    call = "darb_muon_create"
    torch = _torch or _load_torch()
    params, m = list(params), list(m)
    copies = None if copies is None else list(copies)
    n = len(params)
    if len(m) != n or (copies is not None and len(copies) != n):
        _refuse(call, "one momentum (and copy) for every parameter")
    grad_dtype = torch.float32 if grad_dtype is None else grad_dtype
    if grad_dtype not in (torch.float32, torch.bfloat16):
        _refuse(call, "grad_dtype must be float32 or bfloat16")
    for name, tensors, dtype in (("params", params, torch.float32), ("m", m, torch.float32), ("copies", copies or (), torch.bfloat16)):
        for t, p in zip(tensors, params):
            if t is None and name == "copies":
                continue
            if t.dim() != 2 or not t.is_cuda or t.dtype != dtype or t.shape != p.shape or not t.is_contiguous():
                _refuse(call, f"{name} must be contiguous CUDA matrices of {dtype}, of the parameters' shapes")
    array = lambda ts: (ctypes.c_void_p * n)(*[None if t is None else t.data_ptr() for t in ts])  # noqa: E731
    sides = [(ctypes.c_int64 * n)(*[p.shape[i] for p in params]) for i in range(2)]
    out = ctypes.c_void_p()
    _check(lib().darb_muon_create(n, *sides, array(params), array(m), None if copies is None else array(copies),
                                  BF16 if grad_dtype == torch.bfloat16 else F32, ctypes.byref(out), _stream(stream)), call)
    return Muon(out.value, [params, m, copies], [p.shape for p in params], grad_dtype)


def darb_muon_step(plan: Muon, grads, lr: float, beta: float = 0.95, weight_decay: float = 0.01, eps: float = 1e-7,
                   nesterov: bool = True, grad_scale=None, stream=None):
    """One step with the gradients `grads` of the plan's matrices, of their shapes (None: that matrix is left as it
    is).  grad_scale: float32 CUDA scalar that multiplies every gradient."""
    call = "darb_muon_step"
    pointers = _gradient_pointers(plan, grads, call)
    for i, (g, shape) in enumerate(zip(grads, plan.shapes)):   # rows and columns matter here
        if g is not None and g.shape != shape:
            _refuse(call, f"gradient {i} must have its matrix's shape")
    _check(lib().darb_muon_step(plan.ptr, pointers, _vector(grad_scale, 1, (_torch or _load_torch()).float32, call, "grad_scale"),
                                lr, beta, weight_decay, eps, bool(nesterov), _stream(stream)), call)


def darb_muon_sync_status(plan: Muon, stream=None):
    """Synchronise and raise if a step's bounded wait gave up."""
    _check(lib().darb_muon_sync_status(plan.ptr, _stream(stream)), "darb_muon_sync_status")


def darb_muon_destroy(plan: Muon | None):
    if plan is None or plan.ptr is None:
        return
    _check(lib().darb_muon_destroy(plan.ptr), "darb_muon_destroy")
    plan.ptr = None
