"""Beam search over the logits of a head (C ABI in ``include/seedq_beam.h``): one step's
selection over beams and vocabulary, and the beams' states moved to those that continue
them.

Every function of the C ABI has a wrapper of the same name that only marshals
arguments. The helpers (``beam_select``, ``beam_reorder``) check their tensors, allocate
the outputs and the workspace and call the same functions directly; with ``stream``
given they allocate on that stream too. All of them are in the package's own
namespace. They stand outside autograd.
"""
from __future__ import annotations

import ctypes
import functools
import math
from dataclasses import dataclass

import numpy as np

from . import _check, _ptr, _stream
from . import lib as _base_lib
from .ops import _logits, _on, _rows, _same, _type

SEEDQ_MAX_BEAMS = 32
SEEDQ_MAX_BEAM_TOP = 32
SEEDQ_MAX_BEAM_STATES = 4096

_lib = None
torch = _handle = _current_device = None   # from the first call on


class BeamState(ctypes.Structure):
    _fields_ = [("d_src", ctypes.c_void_p), ("d_dst", ctypes.c_void_p), ("src_row", ctypes.c_int64),
                ("dst_row", ctypes.c_int64), ("src_outer", ctypes.c_int64),
                ("dst_outer", ctypes.c_int64), ("outer", ctypes.c_int64), ("inner", ctypes.c_int64)]


def lib() -> ctypes.CDLL:
    global _lib, torch, _handle, _current_device
    if _lib is None:
        import torch
        _handle, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        L = _base_lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.seedq_beam_select_workspace_bytes.restype = sz
        L.seedq_beam_select_workspace_bytes.argtypes = [i64, i32, i64, i32]
        L.seedq_beam_select.restype = ctypes.c_int
        L.seedq_beam_select.argtypes = [vp, i32, i64, i64, i32, i64, vp, vp, i64, i32, vp, vp, vp, vp, sz,
                                        vp]
        L.seedq_beam_reorder.restype = ctypes.c_int
        L.seedq_beam_reorder.argtypes = [vp, i64, vp, i64, i32, i32, vp]
        _lib = L
    return _lib


# ---------------------------------------------------------------- C ABI wrappers

def seedq_beam_select_workspace_bytes(batch: int, beams: int, vocab: int, top: int) -> int:
    return int(lib().seedq_beam_select_workspace_bytes(batch, beams, vocab, top))


def seedq_beam_select(d_logits, type: int, ld: int, batch: int, beams: int, vocab: int, d_scores,
                      d_finished, pad_token: int, top: int, d_score, d_parent, d_token,
                      d_workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    _check(lib().seedq_beam_select(_ptr(d_logits), type, ld, batch, beams, vocab, _ptr(d_scores),
                                   _ptr(d_finished), pad_token, top, _ptr(d_score), _ptr(d_parent),
                                   _ptr(d_token), _ptr(d_workspace), workspace_bytes,
                                   _stream(stream)), "seedq_beam_select")


def seedq_beam_reorder(states, nstates: int, d_parent, batch: int, in_beams: int, out_beams: int,
                       stream=None) -> None:
    """states: a ctypes array of BeamState."""
    _check(lib().seedq_beam_reorder(states, nstates, _ptr(d_parent), batch, in_beams, out_beams,
                                    _stream(stream)), "seedq_beam_reorder")


# ---------------------------------------------------------------- helpers

_select_workspace = functools.lru_cache(maxsize=256)(seedq_beam_select_workspace_bytes)


@dataclass
class BeamStep:
    """The continuations of ``beam_select``, [batch, top] each, the best first: score
    fp32, parent (the beam in its sequence) and token int64. Where there are none left
    score is -inf, parent and token -1."""
    score: object
    parent: object
    token: object


def beam_select(logits, scores, top: int, finished=None, pad_token: int = 0, stream=None) -> BeamStep:
    """The ``top`` best continuations of each sequence over its beams and the
    vocabulary: logits (torch fp32, fp16 or bf16 [batch * beams, vocab] on the GPU),
    scores fp32 [batch, beams] (the log probabilities so far, -inf for a dead beam).
    A beam that is ``finished`` (bool or uint8 [batch, beams]) is continued by pad_token
    alone, at its own score."""
    L = _lib or lib()
    t, device = _type(logits.dtype, "logits"), logits.get_device()
    shape = logits.shape
    if device < 0 or device != _current_device() or len(shape) != 2 or shape[1] < 1:
        _logits(logits, "logits")   # names what is wrong
    nrows, vocab = shape
    shape = scores.shape
    if len(shape) != 2 or not 1 <= shape[1] <= SEEDQ_MAX_BEAMS:
        raise ValueError(f"scores: [batch, 1 to {SEEDQ_MAX_BEAMS} beams] wanted, not {tuple(shape)}")
    batch, beams = shape
    if nrows != batch * beams:
        raise ValueError(f"logits: {batch * beams} rows wanted, not {nrows}")
    if not 1 <= top <= SEEDQ_MAX_BEAM_TOP:
        raise ValueError(f"top: 1 to {SEEDQ_MAX_BEAM_TOP} wanted, not {top}")
    _same(scores, device, shape, torch.float32, "scores")
    if finished is not None:
        _same(finished, device, shape, torch.bool if finished.dtype == torch.bool else torch.uint8,
              "finished")
        if pad_token < 0:
            raise ValueError(f"pad_token: not negative wanted, not {pad_token}")
    if stream is None:
        return _select(L, logits, t, device, scores, batch, beams, vocab, top, finished, pad_token)
    with _on(stream):
        return _select(L, logits, t, device, scores, batch, beams, vocab, top, finished, pad_token)


def _select(L, logits, t, device, scores, batch, beams, vocab, top, finished, pad_token):
    x, ld = _rows(logits)
    score = scores.new_empty((batch, top))
    parent = x.new_empty((batch, top), dtype=torch.int64)
    token = torch.empty_like(parent)
    nws = _select_workspace(batch, beams, vocab, top)
    ws = x.new_empty(nws, dtype=torch.uint8)
    _check(L.seedq_beam_select(x.data_ptr(), t, ld, batch, beams, vocab, scores.data_ptr(),
                               None if finished is None else finished.data_ptr(), pad_token, top,
                               score.data_ptr(), parent.data_ptr(), token.data_ptr(), ws.data_ptr(), nws,
                               _handle(device)), "seedq_beam_select")
    return BeamStep(score, parent, token)


def _pieces(shape, stride, size: int):
    """(row stride, pieces, stride of pieces, bytes of a piece) of rows in bytes, or None
    where a row is more than pieces at one stride."""
    inner, outer, step, i = size, 1, 0, len(shape) - 1
    while i > 0 and (shape[i] == 1 or stride[i] * size == inner):
        inner *= shape[i]
        i -= 1
    while i > 0:
        if shape[i] != 1:
            at = stride[i] * size
            if outer == 1:
                if at < inner:
                    return None
                step = at
            elif at != outer * step:
                return None
            outer *= shape[i]
        i -= 1
    return stride[0] * size, outer, step, inner


def _split(a, b):
    """a and b with the pieces of the one whose pieces are longer cut to the other's, or
    None where they do not divide them."""
    if a[3] == b[3]:
        return a, b
    if a[3] < b[3]:
        other = _split(b, a)
        return other and (other[1], other[0])
    row, outer, step, inner = a
    if inner % b[3] or (outer > 1 and step != inner):
        return None
    return (row, outer * (inner // b[3]), b[3], b[3]), b


@functools.lru_cache(maxsize=1024)
def _moved(shape, stride, to_stride, size: int):
    """How rows of one layout go to another: (source's and destination's row stride,
    source's and destination's stride of pieces, pieces, bytes of a piece), or None;
    to_stride None for dense rows."""
    src = _pieces(shape, stride, size)
    if to_stride is None:
        n = size
        for k in shape[1:]:
            n *= k
        dst = (n, 1, 0, n)
    else:
        dst = _pieces(shape, to_stride, size)
    both = src and dst and _split(src, dst)
    if not both:
        return None
    src, dst = both
    return src[0], dst[0], src[2], dst[2], src[1], src[3]


class _Bytes:
    """Bytes that numpy compares the addresses of and never reads."""

    def __init__(self, start, shape, strides):
        self.__array_interface__ = {"version": 3, "typestr": "|u1", "data": (start, False), "shape": shape,
                                    "strides": strides}


def _meet(intervals) -> bool:
    """Whether one of the intervals (start, end, written) that is written meets another."""
    end = end_written = -1   # of those that start before
    for lo, hi, written in sorted(intervals):
        if lo < (end if written else end_written):
            return True
        end = max(end, hi)
        if written:
            end_written = max(end_written, hi)
    return False


def _races(regions) -> bool:
    """Whether one of the regions that is written shares a byte with another one. A region: (start,
    stride of rows, rows, stride of pieces, pieces, bytes of a piece, written)."""
    regions = sorted(regions)
    ends = [at + (rows - 1) * row + (outer - 1) * step + inner
            for at, row, rows, step, outer, inner, _ in regions]
    first, end = 0, -1
    for i, hi in enumerate(ends):   # those from first on lie in one stretch of memory
        if regions[i][0] >= end:
            if i - first > 1 and _races_near(regions[first:i], ends[first:i]):
                return True
            first = i
        if hi > end:
            end = hi
    return len(ends) - first > 1 and _races_near(regions[first:], ends[first:])


def _races_near(regions, ends) -> bool:
    if not _meet([(r[0], end, r[6]) for r, end in zip(regions, ends)]):
        return False
    # Between each other's rows or pieces (the layers of one tensor): their places modulo a
    # number that every stride is a multiple of.
    by_row = math.gcd(*(row for _, row, rows, _, _, _, _ in regions if rows > 1))
    by_piece = math.gcd(by_row, *(step for _, _, _, step, outer, _, _ in regions if outer > 1))
    for by, whole in ((by_row, True), (by_piece, False)):
        places = []
        for at, _, _, step, outer, inner, written in regions:
            n = inner + ((outer - 1) * step if whole else 0)
            if by and n <= by:
                at %= by
                places += (at, at + n, written), (0, at + n - by, written)   # what goes on at the front
        if len(places) == 2 * len(regions) and not _meet([p for p in places if p[0] < p[1]]):
            return False
    base = regions[0][0] - 1   # numpy takes no address 0
    arrays = [(np.asarray(_Bytes(at - base, (rows, outer, inner), (row, step, 1))), written)
              for at, row, rows, step, outer, inner, written in regions]
    try:
        return any(np.shares_memory(a, b, max_work=100000) for i, (a, v) in enumerate(arrays)
                   for b, w in arrays[:i] if v or w)
    except np.exceptions.TooHardError:
        return True


def beam_reorder(states, parents, out=None, stream=None):
    """The states of the beams that continue: row (i, j) of each result is row
    (i, parents[i, j]) of its tensor, zeros for a parent that is none of the sequence's.

    states: a tensor or a list of tensors of any type on the GPU, [batch * beams, ...]
    each with the same number of rows; a row may be a part of a larger cache (a view).
    parents: int64 [batch, out_beams]. ``out``: tensors of the results' shapes and the
    states' types, or the states themselves, whose rows are then moved in place (those that
    are their own parents stay untouched); one that shares memory with another result, another
    state or the parents is refused. Returns a tensor or a list like states."""
    L = _lib or lib()
    single = isinstance(states, torch.Tensor)
    states = [states] if single else list(states)
    if parents.dim() != 2 or not 1 <= parents.shape[1] <= SEEDQ_MAX_BEAMS:
        raise ValueError(f"parents: [batch, 1 to {SEEDQ_MAX_BEAMS}] wanted, not {tuple(parents.shape)}")
    if len(states) > SEEDQ_MAX_BEAM_STATES:
        raise ValueError(f"states: {SEEDQ_MAX_BEAM_STATES} at the most, not {len(states)}")
    batch, out_beams = parents.shape
    device = parents.get_device()
    if device < 0 or device != _current_device():
        raise ValueError(f"parents: on {parents.device}, not on the current GPU")
    _same(parents, device, (batch, out_beams), torch.int64, "parents")
    if out is not None:
        out = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(out) != len(states):
            raise ValueError(f"out: {len(states)} tensors wanted, not {len(out)}")
    rows = states[0].shape[0] if states and states[0].dim() else 0
    beams = rows // batch if batch else 1
    if states and (rows != batch * beams or not 1 <= beams <= SEEDQ_MAX_BEAMS):
        raise ValueError(f"states: rows of {batch} sequences of 1 to {SEEDQ_MAX_BEAMS} beams wanted, "
                         f"not {rows}")
    args = (L, states, parents, out, rows, batch, beams, out_beams, device)
    if stream is None:
        results = _reorder(*args)
    else:
        with _on(stream):
            results = _reorder(*args)
    return results[0] if single else results


def _reorder(L, states, parents, out, rows, batch, beams, out_beams, device):
    out_rows, same = batch * out_beams, beams == out_beams
    new, dense = torch.empty_like, torch.contiguous_format
    results, fields, keep = [], [], []
    for k, s in enumerate(states):
        shape = s.shape
        if not shape or shape[0] != rows or s.get_device() != device:
            raise ValueError(f"states: tensors of {rows} rows on GPU {device} wanted, not "
                             f"{tuple(shape)} on {s.device}")
        if s.is_conj() or s.is_neg():   # memory does not hold its values
            s = s.resolve_conj().resolve_neg()
            keep.append(s)
        if out is None:
            o, to = (new(s, memory_format=dense) if same else s.new_empty((out_rows, *shape[1:]))), None
        else:
            o = out[k]
            if o.is_conj() or o.is_neg():
                raise ValueError("out: tensors whose memory holds their values wanted")
            if o.dtype != s.dtype or o.shape != (out_rows, *shape[1:]) or o.get_device() != device:
                raise ValueError(f"out: {s.dtype} of shape {(out_rows, *shape[1:])} on GPU {device} "
                                 f"wanted, not {o.dtype} {tuple(o.shape)} on {o.device}")
            to = o.stride()
            if _pieces(o.shape, to, 1) is None:
                raise ValueError("out: rows that are pieces at one stride wanted")
        results.append(o)
        at, to_at = s.data_ptr(), o.data_ptr()
        if not at or not to_at:   # no elements
            continue
        if at == to_at and (s.stride() != to or out_beams != beams):
            raise ValueError("out: in place, the states' own layout and number of beams wanted")
        moved = _moved(shape, s.stride(), to, s.element_size())
        if moved is None:
            s = s.contiguous()
            keep.append(s)
            at, moved = s.data_ptr(), _moved(shape, s.stride(), to, s.element_size())
        fields += (at, to_at, *moved)
    if out is not None and fields:
        regions = [(parents.data_ptr(), 0, 1, 0, 1, 8 * out_rows, False)]
        for i in range(0, len(fields), 8):
            at, to_at, row, to_row, step, to_step, outer, inner = fields[i:i + 8]
            regions.append((to_at, to_row, out_rows, to_step, outer, inner, True))
            if at != to_at:
                regions.append((at, row, rows, step, outer, inner, False))
        if _races(regions):
            raise ValueError("out: tensors that share no memory with another result, another state or the "
                             "parents wanted")
    if fields:
        array = (ctypes.c_int64 * len(fields))(*fields)   # BeamStates
        _check(L.seedq_beam_reorder(array, len(fields) // 8, parents.data_ptr(), batch, beams,
                                    out_beams, _handle(device)), "seedq_beam_reorder")
    if out is not None:
        torch.autograd.graph.increment_version(results)   # written, as autograd counts it
    return results
