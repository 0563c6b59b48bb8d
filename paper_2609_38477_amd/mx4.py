"""Matrices of microscaled 4-bit floats (C ABI in ``include/seedq_mx4.h``): quantise,
dequantise, products with vectors in 16 or 32 bits and products of two coded matrices
on the matrix core.

Every function of the C ABI has a wrapper of the same name that only marshals
arguments. The helpers (``mx4_quantize``, ``mx4_dequantize``, ``mx4_gemv``,
``mx4_matmul``) check their tensors, allocate the outputs and the workspace and call
the same functions directly; with ``stream`` given they allocate on that stream too.
All of them are in the package's own namespace. They stand outside autograd.
"""
from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass

from . import _check, _ptr, _stream
from . import lib as _base_lib
from .ops import SEEDQ_F32, _device, _on, _rows, _same, _type

BLOCK = 32

_lib = None
torch = _handle = _current_device = None   # from the first call on


def lib() -> ctypes.CDLL:
    global _lib, torch, _handle, _current_device
    if _lib is None:
        import torch
        _handle, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        L = _base_lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.seedq_mx4_row_words.restype = sz
        L.seedq_mx4_row_words.argtypes = [i64]
        L.seedq_mx4_quantize.restype = ctypes.c_int
        L.seedq_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
        L.seedq_mx4_dequantize.restype = ctypes.c_int
        L.seedq_mx4_dequantize.argtypes = [vp, vp, i64, i64, vp, i32, i64, vp]
        L.seedq_mx4_gemv_workspace_bytes.restype = sz
        L.seedq_mx4_gemv_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.seedq_mx4_gemv.restype = ctypes.c_int
        L.seedq_mx4_gemv.argtypes = [vp, vp, i64, i64, i64, vp, i32, i64, vp, i32, i64, vp, sz, vp]
        L.seedq_mx4_matmul_workspace_bytes.restype = sz
        L.seedq_mx4_matmul_workspace_bytes.argtypes = [i64, i64, i64]
        L.seedq_mx4_matmul.restype = ctypes.c_int
        L.seedq_mx4_matmul.argtypes = [vp, vp, i64, vp, vp, i64, i64, vp, i32, i64, vp, sz, vp]
        _lib = L
    return _lib


# ---------------------------------------------------------------- C ABI wrappers

def seedq_mx4_row_words(ncols: int) -> int:
    return int(lib().seedq_mx4_row_words(ncols))


def seedq_mx4_quantize(d_W, type: int, ldw: int, nrows: int, ncols: int, d_codes, d_scale,
                       stream=None) -> None:
    _check(lib().seedq_mx4_quantize(_ptr(d_W), type, ldw, nrows, ncols, _ptr(d_codes), _ptr(d_scale),
                                    _stream(stream)), "seedq_mx4_quantize")


def seedq_mx4_dequantize(d_codes, d_scale, nrows: int, ncols: int, d_W_hat, type: int, ldw: int,
                         stream=None) -> None:
    _check(lib().seedq_mx4_dequantize(_ptr(d_codes), _ptr(d_scale), nrows, ncols, _ptr(d_W_hat), type,
                                      ldw, _stream(stream)), "seedq_mx4_dequantize")


def seedq_mx4_gemv_workspace_bytes(nrows: int, ncols: int, nvec: int, xtype: int) -> int:
    return int(lib().seedq_mx4_gemv_workspace_bytes(nrows, ncols, nvec, xtype))


def seedq_mx4_gemv(d_codes, d_scale, nrows: int, ncols: int, nvec: int, d_x, xtype: int, ldx: int,
                   d_y, ytype: int, ldy: int, d_workspace=None, workspace_bytes: int = 0,
                   stream=None) -> None:
    _check(lib().seedq_mx4_gemv(_ptr(d_codes), _ptr(d_scale), nrows, ncols, nvec, _ptr(d_x), xtype, ldx,
                                _ptr(d_y), ytype, ldy, _ptr(d_workspace), workspace_bytes,
                                _stream(stream)), "seedq_mx4_gemv")


def seedq_mx4_matmul_workspace_bytes(na: int, nb: int, ncols: int) -> int:
    return int(lib().seedq_mx4_matmul_workspace_bytes(na, nb, ncols))


def seedq_mx4_matmul(d_a_codes, d_a_scale, na: int, d_b_codes, d_b_scale, nb: int, ncols: int, d_y,
                     ytype: int, ldy: int, d_workspace=None, workspace_bytes: int = 0,
                     stream=None) -> None:
    _check(lib().seedq_mx4_matmul(_ptr(d_a_codes), _ptr(d_a_scale), na, _ptr(d_b_codes),
                                  _ptr(d_b_scale), nb, ncols, _ptr(d_y), ytype, ldy, _ptr(d_workspace),
                                  workspace_bytes, _stream(stream)), "seedq_mx4_matmul")


# ---------------------------------------------------------------- helpers

_gemv_workspace = functools.lru_cache(maxsize=256)(seedq_mx4_gemv_workspace_bytes)
_matmul_workspace = functools.lru_cache(maxsize=256)(seedq_mx4_matmul_workspace_bytes)


@dataclass
class Mx4Weights:
    """A matrix of microscaled 4-bit floats: codes int32 [nrows, row_words], padded with
    zeros, and scale uint8 [nrows, nblocks], the biased exponents of the blocks of 32
    columns (255: NaN)."""
    codes: object
    scale: object
    nrows: int
    ncols: int


def _check_mx4(q: Mx4Weights, what: str) -> int:
    """The device of q, whose tensors are what its sizes say."""
    codes, scale, nrows = q.codes, q.scale, q.nrows
    blocks = (q.ncols + 31) // 32
    device = codes.get_device()
    if device < 0 or device != _current_device() or codes.dtype != torch.int32 \
            or codes.shape != (nrows, 4 * blocks) or not codes.is_contiguous() or scale.dtype != torch.uint8 \
            or scale.shape != (nrows, blocks) or not scale.is_contiguous() or scale.get_device() != device:
        device = _device(codes, what + "codes")     # names what is wrong
        _same(codes, device, (nrows, 4 * blocks), torch.int32, what + "codes")
        _same(scale, device, (nrows, blocks), torch.uint8, what + "scale")
    return device


def _with(stream, f, *args):
    """f(*args), allocating and launching on a stream."""
    if stream is None:
        return f(*args)
    with _on(stream):
        return f(*args)


def mx4_quantize(W, stream=None) -> Mx4Weights:
    """Microscaled 4-bit floats of W (torch fp32, fp16 or bf16 [nrows, ncols] on the
    GPU): for each block of 32 columns the exponent of its largest weight, codes rounded
    to the nearest."""
    L = _lib or lib()
    t = _type(W.dtype, "W")
    if W.dim() != 2:
        raise ValueError(f"W: two dimensions wanted, not {W.dim()}")
    device = W.get_device()
    if device < 0 or device != _current_device():
        _device(W, "W")   # names what is wrong
    return _with(stream, _quantize, L, W, t, device)


def _quantize(L, W, t, device):
    nrows, ncols = W.shape
    blocks = (ncols + 31) // 32
    W, ldw = _rows(W)
    codes = W.new_empty((nrows, 4 * blocks), dtype=torch.int32)
    scale = W.new_empty((nrows, blocks), dtype=torch.uint8)
    _check(L.seedq_mx4_quantize(W.data_ptr(), t, ldw, nrows, ncols, codes.data_ptr(), scale.data_ptr(),
                                _handle(device)), "seedq_mx4_quantize")
    return Mx4Weights(codes, scale, nrows, ncols)


def mx4_dequantize(q: Mx4Weights, dtype=None, stream=None):
    """The weights [nrows, ncols] that q stands for, in dtype (fp32 by default)."""
    L = _lib or lib()
    dtype = torch.float32 if dtype is None else dtype
    t = _type(dtype, "dtype")
    return _with(stream, _dequantize, L, q, dtype, t, _check_mx4(q, ""))


def _dequantize(L, q, dtype, t, device):
    nrows, ncols = q.nrows, q.ncols
    W = q.codes.new_empty((nrows, ncols), dtype=dtype)
    _check(L.seedq_mx4_dequantize(q.codes.data_ptr(), q.scale.data_ptr(), nrows, ncols, W.data_ptr(), t,
                                  ncols, _handle(device)), "seedq_mx4_dequantize")
    return W


def mx4_gemv(q: Mx4Weights, x, out_dtype=None, stream=None):
    """y = W_hat x for the rows x of [nvec, ncols] (or one vector [ncols]), any nvec;
    y [nvec, nrows] (or [nrows]) in out_dtype: x's type (the default) or fp32."""
    L = _lib or lib()
    dtype = x.dtype
    yt = xt = _type(dtype, "x")
    if out_dtype is None:
        out_dtype = dtype
    elif out_dtype != dtype:
        yt = _type(out_dtype, "out_dtype")
        if yt != SEEDQ_F32:
            raise TypeError(f"out_dtype: {dtype} or float32 wanted, not {out_dtype}")
    shape = x.shape
    single = len(shape) == 1
    if len(shape) not in (1, 2) or shape[-1] != q.ncols:
        raise ValueError(f"x: [{q.ncols}] or [nvec, {q.ncols}] wanted, not {tuple(shape)}")
    device = _check_mx4(q, "")
    if x.get_device() != device:
        raise ValueError(f"x: on {x.device}, the codes on {q.codes.device}")
    y = _with(stream, _gemv, L, q, x.unsqueeze(0) if single else x, xt, out_dtype, yt, device)
    return y[0] if single else y


def _gemv(L, q, x, xt, out_dtype, yt, device):
    nrows, ncols = q.nrows, q.ncols
    x, ldx = _rows(x)
    nvec = x.shape[0]
    y = x.new_empty((nvec, nrows), dtype=out_dtype)
    nws = _gemv_workspace(nrows, ncols, nvec, xt)
    ws = x.new_empty(nws, dtype=torch.uint8) if nws else None
    _check(L.seedq_mx4_gemv(q.codes.data_ptr(), q.scale.data_ptr(), nrows, ncols, nvec, x.data_ptr(), xt,
                            ldx, y.data_ptr(), yt, nrows, ws.data_ptr() if nws else None, nws,
                            _handle(device)), "seedq_mx4_gemv")
    return y


def mx4_matmul(a: Mx4Weights, b: Mx4Weights, out_dtype=None, stream=None):
    """A_hat B_hat^T [a.nrows, b.nrows] of two coded matrices with the same number of
    columns (coded vectors and a coded layer), in out_dtype (fp32 by default)."""
    L = _lib or lib()
    out_dtype = torch.float32 if out_dtype is None else out_dtype
    yt = _type(out_dtype, "out_dtype")
    device = _check_mx4(b, "b.")
    if a.ncols != b.ncols:
        raise ValueError(f"a: {b.ncols} columns wanted, not {a.ncols}")
    if a.codes.get_device() != device:
        raise ValueError(f"a: on {a.codes.device}, b on {b.codes.device}")
    _check_mx4(a, "a.")
    return _with(stream, _matmul, L, a, b, out_dtype, yt, device)


def _matmul(L, a, b, out_dtype, yt, device):
    na, nb, ncols = a.nrows, b.nrows, b.ncols
    y = b.codes.new_empty((na, nb), dtype=out_dtype)
    nws = _matmul_workspace(na, nb, ncols)
    ws = y.new_empty(nws, dtype=torch.uint8) if nws else None
    _check(L.seedq_mx4_matmul(a.codes.data_ptr(), a.scale.data_ptr(), na, b.codes.data_ptr(),
                              b.scale.data_ptr(), nb, ncols, y.data_ptr(), yt, nb,
                              ws.data_ptr() if nws else None, nws, _handle(device)), "seedq_mx4_matmul")
    return y
