"""Binding of the state store and its attention (include/lorann_states.h): argument marshalling only, everything runs inside the HIP library.

Tensors live on the GPU and are handed over as pointers with their strides; nothing is copied or converted here, a tensor of another type or
layout than asked for is refused.  Work is enqueued on torch's current stream of the current device and the calls return.

There are no gradients: the store holds rounded codes.  An answer to queries (or scores) that require one can be used forwards, a backward pass that
reaches it raises; what is written into the store is cut off from its graph, as a cast to integers is.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import LorannError, lib as _base_lib

F32, F16, BF16 = 0, 1, 2
MIN_PAGE, MAX_PAGE, MAX_DIM, MAX_HEADS, MAX_FOUND = 16, 256, 128, 1024, 4096
EXPORTS = ["lorann_states_write", "lorann_states_read", "lorann_attend_chunk", "lorann_attend_passages", "lorann_attend_workspace"]

_TYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


class CStates(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("pages", C.c_int64), ("heads", C.c_int32), ("page_size", C.c_int32), ("dim", C.c_int32)]


class CQuestions(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("type", C.c_int32), ("heads", C.c_int32), ("tokens", C.c_int64), ("sequences", C.c_int64),
                ("q_token", C.c_int64), ("q_head", C.c_int64), ("out_token", C.c_int64), ("out_head", C.c_int64), ("q_start", C.c_void_p), ("scale", C.c_float)]


_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        L = _base_lib()
        vp, i32, i64, st, qs = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(CStates), C.POINTER(CQuestions)
        L.lorann_states_write.restype = C.c_int
        L.lorann_states_write.argtypes = [st, vp, vp, i32, i64, i64, i64, i64, i64, vp, vp]
        L.lorann_states_read.restype = C.c_int
        L.lorann_states_read.argtypes = [st, vp, i64, vp, vp, i32, i64, i64, i64, i64, vp]
        L.lorann_attend_chunk.restype = C.c_int
        L.lorann_attend_chunk.argtypes = [st, qs, vp, i32, vp, vp, i64, vp]
        L.lorann_attend_passages.restype = C.c_int
        L.lorann_attend_passages.argtypes = [st, qs, vp, i32, vp, C.c_float, vp, i32, vp, i64, vp, i64, vp]
        L.lorann_attend_workspace.restype = C.c_int64
        L.lorann_attend_workspace.argtypes = [st, qs, i32, i32]
        _lib = L
    return _lib


def _raise(code: int):
    raise LorannError(code, lib().lorann_last_error().decode())


def _array(t, dtype, shape, what):
    """The address of a contiguous tensor of this type and shape."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be a {dtype} tensor of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous (no copy is made)")
    return t.data_ptr()


def _strides(x, what):
    token, head, value = x.stride()
    if value != 1 and x.shape[2] > 1:
        raise ValueError(f"{what}: the values of a row must be consecutive")
    return token, head


class _NoGradient(torch.autograd.Function):
    """The answer as it is, in a graph that ends here with an error instead of leaving the inputs' gradients out."""

    @staticmethod
    def forward(ctx, out, *inputs):
        ctx.mark_dirty(out)
        return out

    @staticmethod
    def backward(ctx, grad):
        raise NotImplementedError("attention over the state store has no gradient (the store holds rounded codes): detach its inputs, or call it under torch.no_grad()")


def _no_gradient(out, *inputs):
    if not torch.is_grad_enabled():
        return out
    if out.grad_fn is not None and out.grad_fn.name() == "_NoGradientBackward":       # (a buffer used again: one such end is enough, a chain would grow with every call)
        return out
    return _NoGradient.apply(out, *inputs)


class States:
    """Keys and values of tokens in 8 bits with one step per token and head, in pages.

    k_codes   [pages, heads, page_size, dim] int8       v_codes   [pages, heads, dim, page_size] int8 (transposed inside a page)
    k_scales  [pages, heads, page_size] float32         v_scales  the same
    The tensors stay the caller's; slot = page * page_size + place in the page."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales):
        self.k_codes, self.v_codes, self.k_scales, self.v_scales = k_codes, v_codes, k_scales, v_scales
        if k_codes.dim() != 4:
            raise ValueError(f"k_codes must be [pages, heads, page_size, dim], got {tuple(k_codes.shape)}")
        self.pages, self.heads, self.page_size, self.dim = n, h, p, d = k_codes.shape
        self._gpu = k_codes.device.index if k_codes.is_cuda else None
        steps = (n, h, p)
        if not (k_codes.dtype is torch.int8 and v_codes.dtype is torch.int8 and k_scales.dtype is torch.float32 and v_scales.dtype is torch.float32
                and v_codes.shape == (n, h, d, p) and k_scales.shape == steps and v_scales.shape == steps
                and k_codes.is_contiguous() and v_codes.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()):
            for t, dtype, shape, what in ((k_codes, torch.int8, (n, h, p, d), "k_codes"), (v_codes, torch.int8, (n, h, d, p), "v_codes"),
                                          (k_scales, torch.float32, steps, "k_scales"), (v_scales, torch.float32, steps, "v_scales")):
                _array(t, dtype, shape, what)          # (says which)
        self._st = CStates(k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), n, h, p, d)

    @property
    def device(self):
        return self.k_codes.device

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, dim: int, device="cuda") -> "States":
        """A store of zeros."""
        z = lambda *shape, t: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        return cls(z(pages, heads, page_size, dim, t=torch.int8), z(pages, heads, dim, page_size, t=torch.int8),
                   z(pages, heads, page_size, t=torch.float32), z(pages, heads, page_size, t=torch.float32))

    def _rows(self, x, tokens, what):
        if x.shape != (tokens, self.heads, self.dim):
            raise ValueError(f"{what} must be [{tokens}, {self.heads}, {self.dim}], got {tuple(x.shape)}")
        return _strides(x, what)

    def _stream(self):
        """torch's current stream (its handle alone: the stream object takes longer than a launch)."""
        if self._gpu is None:
            return None            # (host memory: the library refuses it)
        if self._gpu != _current_device():
            raise ValueError(f"the store is on cuda:{self._gpu}, the current device is cuda:{_current_device()}")
        return _raw_stream(self._gpu)

    def write(self, k, v, slots):
        """Quantise keys and values [tokens, heads, dim] (float32, float16 or bfloat16; any distances between tokens and heads) into their slots
        [tokens] int64; a slot outside the store leaves its token out."""
        n = slots.shape[0]
        kt, kh = self._rows(k, n, "k")
        vt, vh = self._rows(v, n, "v")
        if k.dtype != v.dtype or k.dtype not in _TYPE:
            raise ValueError(f"k and v must both be float32, float16 or bfloat16, got {k.dtype} and {v.dtype}")
        rc = lib().lorann_states_write(self._st, k.data_ptr(), v.data_ptr(), _TYPE[k.dtype], n, kt, kh, vt, vh, _array(slots, torch.int64, (n,), "slots"), self._stream())
        if rc:
            _raise(rc)

    def read(self, slots, dtype=torch.bfloat16, out=None):
        """(keys, values) [tokens, heads, dim] of the tokens in slots [tokens] int64, zeros where a slot is outside the store.  out: two tensors to write
        to (any distances between tokens and heads)."""
        n = slots.shape[0]
        if out is None:
            k = torch.empty((n, self.heads, self.dim), dtype=dtype, device=self.k_codes.device)
            v = torch.empty_like(k)
        else:
            k, v = out
        kt, kh = self._rows(k, n, "out[0]")
        vt, vh = self._rows(v, n, "out[1]")
        if k.dtype != v.dtype or k.dtype not in _TYPE:
            raise ValueError(f"keys and values are read as float32, float16 or bfloat16, got {k.dtype} and {v.dtype}")
        rc = lib().lorann_states_read(self._st, _array(slots, torch.int64, (n,), "slots"), n, k.data_ptr(), v.data_ptr(), _TYPE[k.dtype], kt, kh, vt, vh, self._stream())
        if rc:
            _raise(rc)
        return k, v

    def _questions(self, q, q_start, sequences, scale, out):
        tokens, heads, dim = q.shape
        if dim != self.dim:
            raise ValueError(f"q must be [tokens, heads, {self.dim}], got {tuple(q.shape)}")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape or out.dtype is not q.dtype:
            raise ValueError(f"out must be {tuple(q.shape)} {q.dtype}, got {tuple(out.shape)} {out.dtype}")
        qt, qh = _strides(q, "q")
        ot, oh = _strides(out, "out")
        return CQuestions(q.data_ptr(), out.data_ptr(), _TYPE.get(q.dtype, -1), heads, tokens, sequences, qt, qh, ot, oh,
                          None if q_start is None else _array(q_start, torch.int32, (sequences + 1,), "q_start"), dim ** -0.5 if scale is None else scale), out

    def _workspace(self, qs, found, width, workspace):
        if workspace is not None:
            if not workspace.is_contiguous():          # (its size would not be the memory it has)
                raise ValueError("workspace must be contiguous")
            return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace
        need = lib().lorann_attend_workspace(self._st, qs, found, width)
        if need < 0:
            _raise(need)
        if not need:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=self.k_codes.device)
        return workspace.data_ptr(), need, workspace

    def workspace_bytes(self, q, sequences: int, width: int, found: int = 0, ragged: bool = False) -> int:
        """Bytes of `workspace` that a call with these queries and sizes needs (found = 0: attend_chunk; ragged: with q_start)."""
        qs = CQuestions(None, None, _TYPE.get(q.dtype, -1), q.shape[1], q.shape[0], sequences, 0, 0, 0, 0, 1 if ragged else None, 1.0)
        need = lib().lorann_attend_workspace(self._st, qs, found, width)
        if need < 0:
            _raise(need)
        return need

    def attend_chunk(self, q, tables, lengths, q_start=None, scale=None, out=None, workspace=None):
        """Every sequence's newest tokens attend to the sequence's tokens up to and including themselves.

        q [tokens, heads, dim] float16 or bfloat16; tables [sequences, width] int32 page numbers; lengths [sequences] int32 tokens in the store, the new
        ones included; q_start [sequences + 1] int32 first query of each sequence (None: the same number each); scale: dim ** -0.5 by default.
        workspace: a tensor to work in (workspace_bytes), for callers that allocate nothing.  Returns out [tokens, heads, dim]."""
        n, width = tables.shape
        qs, out = self._questions(q, q_start, n, scale, out)
        ws, size, keep = self._workspace(qs, 0, width, workspace)
        rc = lib().lorann_attend_chunk(self._st, qs, _array(tables, torch.int32, (n, width), "tables"), width, _array(lengths, torch.int32, (n,), "lengths"),
                                       ws, size, self._stream())
        if rc:
            _raise(rc)
        return _no_gradient(out, q) if q.requires_grad else out

    def attend_passages(self, q, ids, tables, lengths, q_start=None, scores=None, score_weight=1.0, scale=None, out=None, workspace=None):
        """The queries of each sequence attend to all tokens of the passages found for it.

        ids [sequences, found] int64 passage numbers as Index.search returns them (outside [0, passages): none); tables [passages, width] int32,
        lengths [passages] int32; scores [sequences, found] float32: score_weight * scores is added to the logits of a passage's keys (the
        search's distances with a negative weight).  The rest as in attend_chunk."""
        n, found = ids.shape
        passages, width = tables.shape
        qs, out = self._questions(q, q_start, n, scale, out)
        ws, size, keep = self._workspace(qs, found, width, workspace)
        rc = lib().lorann_attend_passages(self._st, qs, _array(ids, torch.int64, (n, found), "ids"), found,
                                          None if scores is None else _array(scores, torch.float32, (n, found), "scores"), score_weight,
                                          _array(tables, torch.int32, (passages, width), "tables"), width, _array(lengths, torch.int32, (passages,), "lengths"), passages,
                                          ws, size, self._stream())
        if rc:
            _raise(rc)
        return _no_gradient(out, q, scores) if q.requires_grad or (scores is not None and scores.requires_grad) else out
