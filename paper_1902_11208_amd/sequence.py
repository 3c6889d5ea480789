"""Layers along the packed frames of the examples (or any packed tokens):
linear attention with a decay for each head, root-mean-square norm of a
residual sum, dropout, and the attention's single-token step.

Tokens lie example after example without padding, as the output layer's frames
do. Every step of the computation runs in libmdlstm.so's HIP kernels; this
module and its native part (_binding: tensor checks, pointers and strides) own
buffers and marshal arguments. Objects own their output buffers: a call
overwrites what the call before returned. Calls run on `stream` (default: the
current stream), and buffers are allocated for the stream of the call that first
needs them; an object, its tensors and what it returned have to outlive the work
enqueued on any other stream. An object's calls share its buffers and workspace,
so calls on several streams have to be put in order by the caller.
"""
from __future__ import annotations

import contextlib
import ctypes

import numpy as np
import torch

from ._lib import AttentionDesc, NormDesc, lib
from .api import check_tensor, dtype_code

try:
    from . import _binding
except ImportError as e:
    raise RuntimeError("the native binding is missing: build it with `python -m paper_1902_11208_amd.build`") from e

FP8 = torch.float8_e4m3fn


def _stream(stream):
    return None if stream is None else stream.cuda_stream


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory for work on `stream`: what the current stream freed may still be in use there."""
    if stream is not None and not isinstance(stream, torch.cuda.Stream):  # another holder of a stream handle
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _u64(v, name: str) -> int:
    if type(v) is not int:
        v = int(v)
    if not 0 <= v < 1 << 64:
        raise ValueError(f"{name} {v} is not a 64-bit unsigned number")
    return v


def _apart(a: torch.Tensor, b) -> bool:
    """False where two contiguous tensors share memory."""
    return not isinstance(b, torch.Tensor) or (a.data_ptr() + a.nbytes <= b.data_ptr() or
                                               b.data_ptr() + b.nbytes <= a.data_ptr())


class DecayAttention:
    """Linear attention with a decay for each head over packed sequences.

        S_t = exp(-rates[h]) S_{t-1} + k_t v_t^T        o_t = scale q_t^T S_t

    per sequence and head, the state S [dim_k, dim_v] in fp32 restarting at
    every sequence's edge. lengths: tokens of each sequence (host), e.g. the
    widths of an output layer's rectangles; zero is allowed. rates: [heads] fp32
    device tensor, >= 0. kv_heads: heads of k and v, shared by heads / kv_heads
    query heads each. scale: 1 / sqrt(dim_k) unless given. dtype: storage of q, k, v,
    o and their gradients; sums and states are fp32, and outputs are rounded once.

    States that a call returned may be given back to the object, to go through
    sequences piece by piece: a call writes to a buffer that neither its
    arguments nor the forward call it belongs to use. Its other outputs must not
    be its inputs.
    """

    def __init__(self, lengths, heads: int, dim_k: int, dim_v: int, rates: torch.Tensor, dtype=torch.bfloat16,
                 kv_heads: int = None, scale: float = None):
        n = np.asarray(lengths, np.int64).reshape(-1)
        if n.size and n.min() < 0:
            raise ValueError("a sequence has a negative length")
        self.heads, self.kv_heads = int(heads), int(heads if kv_heads is None else kv_heads)
        self.dim_k, self.dim_v, self.dtype = int(dim_k), int(dim_v), dtype
        self.n, self.tokens = int(n.size), int(n.sum())
        self.longest = int(n.max()) if n.size else 0
        desc = AttentionDesc(self.heads, self.kv_heads, self.dim_k, self.dim_v, dtype_code(dtype),
                             float(max(1, self.dim_k) ** -0.5 if scale is None else scale))
        check_tensor(rates, "rates", (self.heads,), torch.float32)
        self.rates, self.device = rates, rates.device
        self._bytes = [int(lib().mdlstm_attention_workspace_bytes(ctypes.byref(desc), self.n, self.tokens, self.longest,
                                                                  b)) for b in (0, 1)]
        if not all(self._bytes):
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        self._state_shape = (self.n, self.heads, self.dim_k, self.dim_v)
        self.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(self.device)
        # longest first, so that no long sequence starts when the others are done
        self.order = torch.from_numpy(np.argsort(-n, kind="stable").astype(np.int32)).to(self.device)
        self._op = _binding.Attention(self.heads, self.kv_heads, self.dim_k, self.dim_v, desc.dtype, desc.scale, self.n,
                                      self.tokens, self.longest, self.offsets, self.order, rates)
        self._ws = [None, None]
        self._o = self._grads = self._saved = None
        self._finals, self._dstates = [], []

    def _spare(self, buffers: list, stream, *used) -> torch.Tensor:
        """The first of the buffers of states that none of `used` lies in."""
        for b in buffers:
            if all(_apart(b, u) for u in used):
                return b
        buffers.append(_empty(self._state_shape, torch.float32, self.device, stream))
        return buffers[-1]

    def _workspace(self, backward: int, stream) -> torch.Tensor:
        if self._ws[backward] is None:
            self._ws[backward] = _empty(self._bytes[backward], torch.uint8, self.device, stream)
        return self._ws[backward]

    def forward(self, q, k, v, state=None, final_state: bool = False, stream=None):
        """o [tokens, heads, dim_v]; with final_state also the states the sequences leave [n, heads, dim_k, dim_v].
        state: the states they start from (None: zero). q, k, v may be views of one projection's output."""
        if self._o is None:
            self._o = _empty((self.tokens, self.heads, self.dim_v), self.dtype, self.device, stream)
        final = self._spare(self._finals, stream, state) if final_state else None
        self._op.forward(q, k, v, state, self._o, final, self._workspace(0, stream), _stream(stream))
        self._saved = (q, k, v, state)
        return (self._o, final) if final_state else self._o

    def backward(self, do, dstate=None, stream=None):
        """(dq, dk, dv) after a forward call, from the gradient of o (and of the final states, dstate); where the
        forward was given states, (dq, dk, dv, gradient of those)."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this layer first")
        q, k, v, state = self._saved
        if self._grads is None:
            self._grads = tuple(_empty((self.tokens, h, d), self.dtype, self.device, stream) for h, d in (
                (self.heads, self.dim_k), (self.kv_heads, self.dim_k), (self.kv_heads, self.dim_v)))
        out = None if state is None else self._spare(self._dstates, stream, state, dstate)
        self._op.backward(q, k, v, state, do, dstate, *self._grads, out, self._workspace(1, stream), _stream(stream))
        return self._grads if state is None else self._grads + (out,)


def decay_attention_step(q, k, v, state, rates, slots=None, scale: float = None, out=None, stream=None) -> torch.Tensor:
    """One token for each of n sequences: q [n, heads, dim_k], k [n, kv_heads, dim_k], v [n, kv_heads, dim_v] advance
    the fp32 states [slots, heads, dim_k, dim_v] in place and give o [n, heads, dim_v]. slots: int32 [n] device
    tensor, the state of each row (None: row i has state i); a slot outside the states marks an idle row, whose o
    is zero. No two rows may name the same slot."""
    return _binding.step(q, k, v, state, rates, slots, scale, out, _stream(stream))


class ResidualNorm:
    """Root-mean-square norm of a residual sum, rows of weight.numel() elements:

        h = residual + dropout(x)        y = h / sqrt(mean(h^2) + eps) * weight

    weight: [cols] fp32 device tensor. dropout: probability of a zero, with the mask of `dropout` (below) for the
    seed and call of the forward; a call number names a draw (a layer's id, the step). out "fp8": y in float8 e4m3
    with a scale for each row, for inference.
    """

    def __init__(self, weight: torch.Tensor, rows: int, dtype=torch.bfloat16, eps: float = 1e-6, dropout: float = 0.0,
                 out: str = None):
        if not isinstance(weight, torch.Tensor) or weight.dim() != 1:
            raise ValueError("weight must be a [cols] tensor")
        if out not in (None, "fp8"):
            raise ValueError(f"out {out!r} is not None or 'fp8'")
        cols = weight.numel()
        check_tensor(weight, "weight", (cols,), torch.float32)
        self.weight, self.rows, self.cols, self.dtype, self.fp8 = weight, int(rows), cols, dtype, out == "fp8"
        self.device = weight.device
        desc = NormDesc(cols, dtype_code(dtype), float(eps), float(dropout))
        nbytes = int(lib().mdlstm_norm_workspace_bytes(ctypes.byref(desc), self.rows))
        if not nbytes:
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        self._op = _binding.Norm(cols, desc.dtype, desc.eps, desc.p, self.rows, weight)
        self._drops = round(float(dropout) * 65536) > 0
        self._ws_bytes, self._ws = nbytes, None
        self._y = self._scale = self._rstd = self._h = self._dx = self._dres = self._dw = self._saved = None

    def forward(self, x, residual=None, seed: int = 0, call: int = 0, stream=None):
        """(y, h), or with out "fp8" (y, scale, h): y[i, j] stands for float(y[i, j]) * scale[i]. h is the new residual;
        without residual and dropout it is x itself (a copy where x is this object's y, which the call overwrites).
        x and residual: [rows, cols], contiguous along their rows."""
        plain = residual is None and not self._drops and (self._y is None or _apart(self._y, x))
        if self._y is None:
            self._y = _empty((self.rows, self.cols), FP8 if self.fp8 else self.dtype, self.device, stream)
            per_row = _empty(self.rows, torch.float32, self.device, stream)
            self._scale, self._rstd = (per_row, None) if self.fp8 else (None, per_row)
        if not plain and self._h is None:
            self._h = _empty((self.rows, self.cols), self.dtype, self.device, stream)
        seed, call = _u64(seed, "seed"), _u64(call, "call")
        self._op.forward(x, residual, None if plain else self._h, self._y, self._scale, self._rstd, seed, call,
                         _stream(stream))
        h = x if plain else self._h
        if self.fp8:
            return self._y, self._scale, h
        self._saved = (h, seed, call, residual is not None)
        return self._y, h

    def backward(self, dy, dh=None, stream=None):
        """(dx, dresidual, dweight) after a forward call, from the gradients of y and of h (dh; None: zero). dresidual
        is None where the forward had no residual, and dx itself without dropout."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this norm first (and no 8-bit output)")
        h, seed, call, residual = self._saved
        if self._dx is None:
            self._dx = _empty((self.rows, self.cols), self.dtype, self.device, stream)
            self._dw = _empty(self.cols, torch.float32, self.device, stream)
            self._ws = _empty(self._ws_bytes, torch.uint8, self.device, stream)
        both = residual and self._drops
        if both and self._dres is None:
            self._dres = _empty((self.rows, self.cols), self.dtype, self.device, stream)
        self._op.backward(h, self._rstd, dy, dh, seed, call, self._dx, self._dres if both else None, self._dw, self._ws,
                          _stream(stream))
        return self._dx, (self._dres if both else self._dx) if residual else None, self._dw


def dropout(x, p: float, seed: int, call: int = 0, residual=None, out=None, stream=None) -> torch.Tensor:
    """residual + dropout(x) (residual None: dropout(x)) with a mask that is never stored: it follows from seed, call
    and an element's place in row-major order alone, so the gradient is the same call on the gradient of the result.
    p is taken to the nearest 2^-16; kept elements are scaled so that the expectation stays. x and residual:
    contiguous, or two-dimensional with contiguous rows. out: contiguous; may be x or residual."""
    return _binding.dropout(x, p, _u64(seed, "seed"), _u64(call, "call"), residual, out, _stream(stream))
