"""Operators beside the seed codec (C ABI in ``include/seedq_ops.h``): weights in
4 bits with group scales, and log probabilities of given tokens with their
gradient.

Every function of the C ABI has a wrapper of the same name that only marshals
arguments. The helpers (``q4_quantize``, ``q4_dequantize``, ``q4_gemv``,
``token_logprobs``, ``token_logprobs_backward``) check their tensors, allocate the
outputs and the workspace and call the same functions directly; with ``stream``
given they allocate on that stream too. All of them are in the package's own
namespace. They stand outside autograd: a result carries no gradient, whatever its
inputs ask for, and ``token_logprobs_backward`` is called by whoever wants one.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
from dataclasses import dataclass

from . import _check, _ptr, _stream
from . import lib as _base_lib

SEEDQ_F32, SEEDQ_F16, SEEDQ_BF16 = 0, 1, 2
SEEDQ_MAX_TOP = 32
SEEDQ_EUNSUPPORTED = -2
GROUPS = (32, 64, 128, 256, 512)

_lib = None
_types = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = _base_lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.seedq_q4_row_words.restype = sz
        L.seedq_q4_row_words.argtypes = [i64]
        L.seedq_q4_quantize.restype = ctypes.c_int
        L.seedq_q4_quantize.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, vp, vp]
        L.seedq_q4_dequantize.restype = ctypes.c_int
        L.seedq_q4_dequantize.argtypes = [vp, vp, vp, i64, i64, i32, vp, i32, i64, vp]
        L.seedq_q4_gemv_workspace_bytes.restype = sz
        L.seedq_q4_gemv_workspace_bytes.argtypes = [i64, i64, i64, i32]
        L.seedq_q4_gemv.restype = ctypes.c_int
        L.seedq_q4_gemv.argtypes = [vp, vp, vp, i64, i64, i32, i64, vp, i32, i64, vp, i32, i64, vp,
                                    sz, vp]
        L.seedq_token_logprobs_workspace_bytes.restype = sz
        L.seedq_token_logprobs_workspace_bytes.argtypes = [i64, i64, i32]
        L.seedq_token_logprobs.restype = ctypes.c_int
        L.seedq_token_logprobs.argtypes = [vp, i32, i64, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp,
                                           sz, vp]
        L.seedq_token_logprobs_backward.restype = ctypes.c_int
        L.seedq_token_logprobs_backward.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp,
                                                    i64, vp]
        _lib = L
    return _lib


# ---------------------------------------------------------------- C ABI wrappers

def seedq_q4_row_words(ncols: int) -> int:
    return int(lib().seedq_q4_row_words(ncols))


def seedq_q4_quantize(d_W, type: int, ldw: int, nrows: int, ncols: int, group: int, d_codes,
                      d_scale, d_zero=None, stream=None) -> None:
    _check(lib().seedq_q4_quantize(_ptr(d_W), type, ldw, nrows, ncols, group, _ptr(d_codes),
                                   _ptr(d_scale), _ptr(d_zero), _stream(stream)),
           "seedq_q4_quantize")


def seedq_q4_dequantize(d_codes, d_scale, d_zero, nrows: int, ncols: int, group: int, d_W_hat,
                        type: int, ldw: int, stream=None) -> None:
    _check(lib().seedq_q4_dequantize(_ptr(d_codes), _ptr(d_scale), _ptr(d_zero), nrows, ncols,
                                     group, _ptr(d_W_hat), type, ldw, _stream(stream)),
           "seedq_q4_dequantize")


def seedq_q4_gemv_workspace_bytes(nrows: int, ncols: int, nvec: int, xtype: int) -> int:
    return int(lib().seedq_q4_gemv_workspace_bytes(nrows, ncols, nvec, xtype))


def seedq_q4_gemv(d_codes, d_scale, d_zero, nrows: int, ncols: int, group: int, nvec: int, d_x,
                  xtype: int, ldx: int, d_y, ytype: int, ldy: int, d_workspace=None,
                  workspace_bytes: int = 0, stream=None) -> None:
    _check(lib().seedq_q4_gemv(_ptr(d_codes), _ptr(d_scale), _ptr(d_zero), nrows, ncols, group,
                               nvec, _ptr(d_x), xtype, ldx, _ptr(d_y), ytype, ldy,
                               _ptr(d_workspace), workspace_bytes, _stream(stream)),
           "seedq_q4_gemv")


def seedq_token_logprobs_workspace_bytes(nrows: int, vocab: int, top: int) -> int:
    return int(lib().seedq_token_logprobs_workspace_bytes(nrows, vocab, top))


def seedq_token_logprobs(d_logits, type: int, ld: int, nrows: int, vocab: int, d_tokens, top: int,
                         d_logprob, d_entropy, d_lse, d_top_token=None, d_top_logprob=None,
                         d_workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    _check(lib().seedq_token_logprobs(_ptr(d_logits), type, ld, nrows, vocab, _ptr(d_tokens), top,
                                      _ptr(d_logprob), _ptr(d_entropy), _ptr(d_lse),
                                      _ptr(d_top_token), _ptr(d_top_logprob), _ptr(d_workspace),
                                      workspace_bytes, _stream(stream)), "seedq_token_logprobs")


def seedq_token_logprobs_backward(d_logits, type: int, ld: int, nrows: int, vocab: int, d_tokens,
                                  d_lse, d_entropy, d_grad_logprob, d_grad_entropy, d_grad_logits,
                                  ldg: int, stream=None) -> None:
    _check(lib().seedq_token_logprobs_backward(_ptr(d_logits), type, ld, nrows, vocab,
                                               _ptr(d_tokens), _ptr(d_lse), _ptr(d_entropy),
                                               _ptr(d_grad_logprob), _ptr(d_grad_entropy),
                                               _ptr(d_grad_logits), ldg, _stream(stream)),
           "seedq_token_logprobs_backward")


# ---------------------------------------------------------------- helpers
#
# A call for one token is bound by the way through these lines, so they take the
# pointers and the stream's handle directly. The workspaces' sizes are functions of the
# arguments below alone.

_gemv_workspace = functools.lru_cache(maxsize=256)(seedq_q4_gemv_workspace_bytes)
_logprobs_workspace = functools.lru_cache(maxsize=256)(seedq_token_logprobs_workspace_bytes)


def _type(dtype, what: str) -> int:
    """The SEEDQ_* code of a torch dtype."""
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: SEEDQ_F32, torch.float16: SEEDQ_F16, torch.bfloat16: SEEDQ_BF16}
    try:
        return _types[dtype]
    except KeyError:
        raise TypeError(f"{what}: float32, float16 or bfloat16 wanted, not {dtype}") from None


def _on(stream):
    """The stream that a helper allocates and launches on; it is one of the current GPU."""
    if stream is None:
        return _current
    import torch
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(stream)
    if stream.device.index != torch.cuda.current_device():
        raise ValueError(f"stream: one of GPU {torch.cuda.current_device()} wanted")
    return torch.cuda.stream(stream)


_current = contextlib.nullcontext()


def _handle(device: int) -> int:
    """Handle of the current stream of a device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


def _device(t, what: str) -> int:
    import torch
    i = t.get_device()
    if i < 0 or i != torch.cuda.current_device():
        raise ValueError(f"{what}: on {t.device}, not on the current GPU")
    return i


def _same(t, device: int, shape, dtype, what: str) -> None:
    """t is a dense tensor of this shape and type on this device."""
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {device} "
                         f"wanted, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows(t):
    """t [n, m] with elements of a row side by side and rows that do not overlap, and
    its row stride."""
    n, m = t.shape
    if t.is_contiguous():
        return t, m
    if (m > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < m):
        return t.contiguous(), m
    return t, (t.stride(0) if n > 1 else m)


@dataclass
class Q4Weights:
    """A matrix in 4 bits: codes int32 [nrows, row_words], scale fp16 and zero uint8
    (or None) [nrows, ngroups]; the value of code u is scale (u - zero), 8 standing
    in for a missing zero point."""
    codes: object
    scale: object
    zero: object
    nrows: int
    ncols: int
    group: int


def _check_q4(q: Q4Weights) -> int:
    """The device of q, whose tensors are what its sizes say."""
    import torch
    codes, zero = q.codes, q.zero
    if q.group not in GROUPS:
        _check(SEEDQ_EUNSUPPORTED, f"Q4Weights: group {q.group}")
    device = _device(codes, "codes")
    groups = (q.nrows, -(-q.ncols // q.group))
    _same(codes, device, (q.nrows, 4 * ((q.ncols + 31) // 32)), torch.int32, "codes")
    _same(q.scale, device, groups, torch.float16, "scale")
    if zero is not None:
        _same(zero, device, groups, torch.uint8, "zero")
    return device


def q4_quantize(W, group: int = 128, zeros: bool = False, stream=None) -> Q4Weights:
    """Round-to-nearest 4-bit codes of W (torch fp32, fp16 or bf16 [nrows, ncols] on
    the GPU) with an fp16 scale, and with ``zeros`` a zero point, for each group of
    columns."""
    import torch
    t = _type(W.dtype, "W")
    if W.dim() != 2:
        raise ValueError(f"W: two dimensions wanted, not {W.dim()}")
    if group not in GROUPS:
        raise ValueError(f"group: one of {GROUPS} wanted, not {group}")
    device = _device(W, "W")
    nrows, ncols = W.shape
    groups = (nrows, -(-ncols // group))
    with _on(stream):
        W, ldw = _rows(W)
        codes = W.new_empty((nrows, 4 * ((ncols + 31) // 32)), dtype=torch.int32)
        scale = W.new_empty(groups, dtype=torch.float16)
        zero = W.new_empty(groups, dtype=torch.uint8) if zeros else None
        _check(lib().seedq_q4_quantize(W.data_ptr(), t, ldw, nrows, ncols, group, codes.data_ptr(),
                                       scale.data_ptr(), _ptr(zero), _handle(device)),
               "seedq_q4_quantize")
    return Q4Weights(codes, scale, zero, nrows, ncols, group)


def q4_dequantize(q: Q4Weights, dtype=None, stream=None):
    """The weights [nrows, ncols] that q stands for, in dtype (fp32 by default)."""
    import torch
    dtype = torch.float32 if dtype is None else dtype
    t = _type(dtype, "dtype")
    device = _check_q4(q)
    nrows, ncols = q.nrows, q.ncols
    with _on(stream):
        W = q.codes.new_empty((nrows, ncols), dtype=dtype)
        _check(lib().seedq_q4_dequantize(q.codes.data_ptr(), q.scale.data_ptr(), _ptr(q.zero), nrows,
                                         ncols, q.group, W.data_ptr(), t, ncols, _handle(device)),
               "seedq_q4_dequantize")
    return W


def q4_gemv(q: Q4Weights, x, out_dtype=None, stream=None):
    """y = W_hat x for the rows x of [nvec, ncols] (or one vector [ncols]), any nvec;
    y [nvec, nrows] (or [nrows]) in out_dtype: x's type (the default) or fp32."""
    import torch
    xt = _type(x.dtype, "x")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    yt = _type(out_dtype, "out_dtype")
    if yt != xt and yt != SEEDQ_F32:
        raise TypeError(f"out_dtype: {x.dtype} or float32 wanted, not {out_dtype}")
    nrows, ncols = q.nrows, q.ncols
    single = x.dim() == 1
    if x.dim() not in (1, 2) or x.shape[-1] != ncols:
        raise ValueError(f"x: [{ncols}] or [nvec, {ncols}] wanted, not {tuple(x.shape)}")
    device = _check_q4(q)
    if x.get_device() != device:
        raise ValueError(f"x: on {x.device}, the codes on {q.codes.device}")
    with _on(stream):
        xx, ldx = _rows(x.unsqueeze(0) if single else x)
        nvec = xx.shape[0]
        y = xx.new_empty((nvec, nrows), dtype=out_dtype)
        nws = _gemv_workspace(nrows, ncols, nvec, xt)
        ws = xx.new_empty(nws, dtype=torch.uint8) if nws else None
        _check(lib().seedq_q4_gemv(q.codes.data_ptr(), q.scale.data_ptr(), _ptr(q.zero), nrows, ncols,
                                   q.group, nvec, xx.data_ptr(), xt, ldx, y.data_ptr(), yt, nrows,
                                   _ptr(ws), nws, _handle(device)), "seedq_q4_gemv")
    return y[0] if single else y


@dataclass
class TokenLogprobs:
    """What ``token_logprobs`` gives for each row of logits (fp32; top_token int64)."""
    logprob: object        # [nrows], or None without tokens
    entropy: object        # [nrows]
    lse: object            # [nrows]: log of the sum of exponentials
    top_token: object      # [nrows, top], or None at top = 0
    top_logprob: object    # [nrows, top], or None at top = 0


def _logits(logits, what: str):
    """Type code and device of rows of logits."""
    t = _type(logits.dtype, what)
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError(f"{what}: [nrows, vocab] wanted, not {tuple(logits.shape)}")
    return t, _device(logits, what)


def token_logprobs(logits, tokens=None, top: int = 0, stream=None) -> TokenLogprobs:
    """Log probability of tokens[t] under the softmax of logits[t] (torch fp32, fp16
    or bf16 [nrows, vocab] on the GPU; tokens int64 [nrows], a negative one asks for
    nothing and gives 0), the entropy, the log of the sum, and the ``top`` likeliest
    tokens with their log probabilities."""
    import torch
    t, device = _logits(logits, "logits")
    nrows, vocab = logits.shape
    if not 0 <= top <= SEEDQ_MAX_TOP:
        raise ValueError(f"top: 0 to {SEEDQ_MAX_TOP} wanted, not {top}")
    if tokens is not None:
        _same(tokens, device, (nrows,), torch.int64, "tokens")
    with _on(stream):
        x, ld = _rows(logits)
        sums = x.new_empty((3, nrows), dtype=torch.float32)
        lse, entropy, logprob = sums.unbind(0)
        if tokens is None:
            logprob = None
        top_token = x.new_empty((nrows, top), dtype=torch.int64) if top else None
        top_logprob = x.new_empty((nrows, top), dtype=torch.float32) if top else None
        nws = _logprobs_workspace(nrows, vocab, top)
        ws = x.new_empty(nws, dtype=torch.uint8) if nws else None
        _check(lib().seedq_token_logprobs(x.data_ptr(), t, ld, nrows, vocab, _ptr(tokens), top,
                                          _ptr(logprob), entropy.data_ptr(), lse.data_ptr(),
                                          _ptr(top_token), _ptr(top_logprob), _ptr(ws), nws,
                                          _handle(device)), "seedq_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, top_token, top_logprob)


def token_logprobs_backward(logits, tokens, lse, entropy=None, grad_logprob=None,
                            grad_entropy=None, out=None, stream=None):
    """Gradient at the logits of sum_t (grad_logprob_t logprob_t + grad_entropy_t
    entropy_t), from what token_logprobs gave; either gradient may be None. ``out``
    (the logits' type and shape) may be the logits themselves."""
    import torch
    t, device = _logits(logits, "logits")
    nrows, vocab = logits.shape
    if grad_logprob is None and grad_entropy is None:
        raise ValueError("grad_logprob or grad_entropy wanted")
    if grad_logprob is not None and tokens is None:
        raise ValueError("grad_logprob needs tokens")
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy needs entropy")
    if tokens is not None:
        _same(tokens, device, (nrows,), torch.int64, "tokens")
    for name, v in (("lse", lse), ("entropy", entropy), ("grad_logprob", grad_logprob),
                    ("grad_entropy", grad_entropy)):
        if v is not None:
            _same(v, device, (nrows,), torch.float32, name)
    with _on(stream):
        x, ld = _rows(logits)
        given = out is not None
        if not given:
            out, ldg = x.new_empty((nrows, vocab)), vocab
        elif out.dtype != x.dtype or out.shape != x.shape or out.get_device() != device \
                or (vocab > 1 and out.stride(1) != 1) or (nrows > 1 and out.stride(0) < vocab):
            raise ValueError("out: the logits' type, shape and device, with dense rows, wanted")
        else:
            ldg = out.stride(0) if nrows > 1 else ld
        _check(lib().seedq_token_logprobs_backward(x.data_ptr(), t, ld, nrows, vocab, _ptr(tokens),
                                                   lse.data_ptr(), _ptr(entropy), _ptr(grad_logprob),
                                                   _ptr(grad_entropy), out.data_ptr(), ldg,
                                                   _handle(device)),
               "seedq_token_logprobs_backward")
    if given:
        torch.autograd.graph.increment_version(out)   # written, as autograd counts it
    return out
