"""Layers along the packed frames of the examples (or any packed tokens):
linear attention with a decay for each head, root-mean-square norm of a
residual sum, dropout, and the attention's single-token step.

Tokens lie example after example without padding, as the output layer's frames
do. Every step of the computation runs in libmdlstm.so's HIP kernels; this
module checks arguments, owns buffers and marshals pointers. Objects own their
output buffers: a call overwrites what the call before returned. Calls run on
`stream` (default: the current stream); an object, its tensors and what it
returned have to outlive the work enqueued on any other stream.
"""
from __future__ import annotations

import ctypes
import functools

import numpy as np
import torch

from ._lib import AttentionDesc, Heads, NormDesc, check, lib
from .api import _ptr, check_tensor, dtype_code

FP8 = torch.float8_e4m3fn
_raw_stream = torch._C._cuda_getCurrentRawStream  # the handle without a Stream object: these calls are short


def _stream(stream, device) -> int:
    return _raw_stream(device.index) if stream is None else stream.cuda_stream


def _complain(t, name: str, shape, dtype: torch.dtype, device):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch.Tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    raise ValueError(f"{name} is on {t.device}, expected {device}")


def _matches(t, name: str, shape, dtype: torch.dtype, device) -> None:
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not dtype or t.device != device:
        _complain(t, name, shape, dtype, device)


def _heads(t, name: str, tokens: int, heads: int, dim: int, dtype: torch.dtype, device) -> Heads:
    """A [tokens, heads, dim] tensor, possibly a view with a contiguous last dimension, as the C ABI takes it."""
    if (not isinstance(t, torch.Tensor) or t.shape != (tokens, heads, dim) or t.dtype is not dtype or
            t.device != device):
        _complain(t, name, (tokens, heads, dim), dtype, device)
    st, sh, sd = t.stride()
    if sd != 1 and dim > 1 and t.numel():
        raise ValueError(f"{name} must be contiguous along its last dimension")
    return Heads(t.data_ptr(), st, sh)


def _full(t, name: str, shape, dtype: torch.dtype, device) -> int:
    """The pointer of a contiguous tensor."""
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not dtype or t.device != device:
        _complain(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


@functools.lru_cache(maxsize=256)
def _attention_desc(heads: int, kv_heads: int, dim_k: int, dim_v: int, dtype: int, scale) -> AttentionDesc:
    return AttentionDesc(heads, kv_heads, dim_k, dim_v, dtype, max(1, dim_k) ** -0.5 if scale is None else scale)


def _rows(t, name: str, shape, dtype: torch.dtype, device) -> int:
    """Stride between the rows of a [rows, cols] tensor that is contiguous along its rows."""
    _matches(t, name, shape, dtype, device)
    rows, cols = shape
    sr, sc = t.stride()
    if rows and cols > 1 and sc != 1:
        raise ValueError(f"{name} must be contiguous along its rows")
    if rows < 2 or cols == 0:
        return cols
    if sr < cols:
        raise ValueError(f"the rows of {name} must not overlap")
    return sr


def _u64(v, name: str) -> int:
    if type(v) is not int:
        v = int(v)
    if not 0 <= v < 1 << 64:
        raise ValueError(f"{name} {v} is not a 64-bit unsigned number")
    return v


class DecayAttention:
    """Linear attention with a decay for each head over packed sequences.

        S_t = exp(-rates[h]) S_{t-1} + k_t v_t^T        o_t = scale q_t^T S_t

    per sequence and head, the state S [dim_k, dim_v] in fp32 restarting at
    every sequence's edge. lengths: tokens of each sequence (host), e.g. the
    widths of an output layer's rectangles; zero is allowed. rates: [heads] fp32
    device tensor, >= 0. kv_heads: heads of k and v, shared by heads / kv_heads
    query heads each. scale: 1 / sqrt(dim_k) unless given.
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
        self.desc = AttentionDesc(self.heads, self.kv_heads, self.dim_k, self.dim_v, dtype_code(dtype),
                                  float(max(1, self.dim_k) ** -0.5 if scale is None else scale))
        check_tensor(rates, "rates", (self.heads,), torch.float32)
        self.rates, self.device = rates, rates.device
        self._bytes = [int(lib().mdlstm_attention_workspace_bytes(ctypes.byref(self.desc), self.n, self.tokens,
                                                                  self.longest, b)) for b in (0, 1)]
        if not all(self._bytes):
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        self._state_shape = (self.n, self.heads, self.dim_k, self.dim_v)
        self.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(self.device)
        # longest first, so that no long sequence starts when the others are done
        self.order = torch.from_numpy(np.argsort(-n, kind="stable").astype(np.int32)).to(self.device)
        self._ws = [None, None]
        self._o = self._final = self._grads = self._dstate = None
        self._saved = None

    def _workspace(self, backward: int) -> torch.Tensor:
        if self._ws[backward] is None:
            self._ws[backward] = torch.empty(self._bytes[backward], dtype=torch.uint8, device=self.device)
        return self._ws[backward]

    def _qkv(self, q, k, v):
        t, dt, dev = self.tokens, self.dtype, self.device
        return (_heads(q, "q", t, self.heads, self.dim_k, dt, dev), _heads(k, "k", t, self.kv_heads, self.dim_k, dt, dev),
                _heads(v, "v", t, self.kv_heads, self.dim_v, dt, dev))

    def _state(self, t, name):
        return None if t is None else _full(t, name, self._state_shape, torch.float32, self.device)

    def forward(self, q, k, v, state=None, final_state: bool = False, stream=None):
        """o [tokens, heads, dim_v]; with final_state also the states the sequences leave [n, heads, dim_k, dim_v].
        state: the states they start from (None: zero). q, k, v may be views of one projection's output."""
        hq, hk, hv = self._qkv(q, k, v)
        pstate = self._state(state, "state")
        if self._o is None:
            self._o = torch.empty((self.tokens, self.heads, self.dim_v), dtype=self.dtype, device=self.device)
        if final_state and self._final is None:
            self._final = torch.empty(self._state_shape, dtype=torch.float32, device=self.device)
        check(lib().mdlstm_attention_forward(self.desc, self.n, self.tokens, self.longest, self.offsets.data_ptr(),
                                             self.order.data_ptr(), self.rates.data_ptr(), hq, hk, hv, pstate, self._o.data_ptr(),
                                             self._final.data_ptr() if final_state else None,
                                             self._workspace(0).data_ptr(), self._bytes[0], _stream(stream, self.device)))
        self._saved = (q, k, v, state)
        return (self._o, self._final) if final_state else self._o

    def backward(self, do, dstate=None, stream=None):
        """(dq, dk, dv) after a forward call, from the gradient of o (and of the final states, dstate); where the
        forward was given states, (dq, dk, dv, gradient of those)."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this layer first")
        q, k, v, state = self._saved
        hq, hk, hv = self._qkv(q, k, v)
        hdo = _heads(do, "do", self.tokens, self.heads, self.dim_v, self.dtype, self.device)
        pdstate = self._state(dstate, "dstate")
        if self._grads is None:
            self._grads = tuple(torch.empty((self.tokens, h, d), dtype=self.dtype, device=self.device) for h, d in (
                (self.heads, self.dim_k), (self.kv_heads, self.dim_k), (self.kv_heads, self.dim_v)))
        if state is not None and self._dstate is None:
            self._dstate = torch.empty(self._state_shape, dtype=torch.float32, device=self.device)
        dq, dk, dv = self._grads
        check(lib().mdlstm_attention_backward(self.desc, self.n, self.tokens, self.longest, self.offsets.data_ptr(),
                                              self.order.data_ptr(), self.rates.data_ptr(), hq, hk, hv, _ptr(state), hdo, pdstate,
                                              dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                              None if state is None else self._dstate.data_ptr(),
                                              self._workspace(1).data_ptr(), self._bytes[1],
                                              _stream(stream, self.device)))
        return self._grads if state is None else self._grads + (self._dstate,)


def decay_attention_step(q, k, v, state, rates, slots=None, scale: float = None, out=None, stream=None) -> torch.Tensor:
    """One token for each of n sequences: q [n, heads, dim_k], k [n, kv_heads, dim_k], v [n, kv_heads, dim_v] advance
    the fp32 states [slots, heads, dim_k, dim_v] in place and give o [n, heads, dim_v]. slots: int32 [n] device
    tensor, the state of each row (None: row i has state i); a slot outside the states marks an idle row, whose o
    is zero. No two rows may name the same slot."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q must be [n, heads, dim_k] and k [n, kv_heads, dim_k]")
    if not isinstance(state, torch.Tensor) or state.dim() != 4:
        raise ValueError("state must be [slots, heads, dim_k, dim_v]")
    (n, heads, dk), kv, dev, dt = q.shape, k.shape[1], q.device, q.dtype
    count, _, _, dv = state.shape
    if not q.is_cuda:
        raise ValueError("q must be a device tensor")
    pstate = _full(state, "state", (count, heads, dk, dv), torch.float32, dev)
    prates = _full(rates, "rates", (heads,), torch.float32, dev)
    pslots = None if slots is None else _full(slots, "slots", (n,), torch.int32, dev)
    desc = _attention_desc(heads, kv, dk, dv, dtype_code(dt), scale)
    hq, hk, hv = (_heads(q, "q", n, heads, dk, dt, dev), _heads(k, "k", n, kv, dk, dt, dev),
                  _heads(v, "v", n, kv, dv, dt, dev))
    if out is None:
        out = torch.empty((n, heads, dv), dtype=dt, device=dev)
    check(lib().mdlstm_attention_step(desc, n, prates, hq, hk, hv, pstate, count, pslots,
                                      _full(out, "out", (n, heads, dv), dt, dev), _stream(stream, dev)))
    return out


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
        self.desc = NormDesc(cols, dtype_code(dtype), float(eps), float(dropout))
        nbytes = int(lib().mdlstm_norm_workspace_bytes(ctypes.byref(self.desc), self.rows))
        if not nbytes:
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        self._drops = round(float(dropout) * 65536) > 0
        shape = (self.rows, cols)
        self._ws_bytes, self._ws = nbytes, None
        self._h = self._dx = self._dres = self._dw = self._saved = None
        if self.fp8:
            self._y = torch.empty(shape, dtype=FP8, device=self.device)
            self._scale = torch.empty(self.rows, dtype=torch.float32, device=self.device)
            self._rstd = None
        else:
            self._y = torch.empty(shape, dtype=dtype, device=self.device)
            self._scale = None
            self._rstd = torch.empty(self.rows, dtype=torch.float32, device=self.device)

    def forward(self, x, residual=None, seed: int = 0, call: int = 0, stream=None):
        """(y, h), or with out "fp8" (y, scale, h): y[i, j] stands for float(y[i, j]) * scale[i]. h is the new residual;
        without residual and dropout it is x itself. x and residual: [rows, cols], contiguous along their rows."""
        shape = (self.rows, self.cols)
        xs = _rows(x, "x", shape, self.dtype, self.device)
        rs = 0 if residual is None else _rows(residual, "residual", shape, self.dtype, self.device)
        plain = residual is None and not self._drops
        if not plain and self._h is None:
            self._h = torch.empty(shape, dtype=self.dtype, device=self.device)
        h = x if plain else self._h
        seed, call = _u64(seed, "seed"), _u64(call, "call")
        y = self._y.data_ptr()
        check(lib().mdlstm_norm_forward(self.desc, self.rows, x.data_ptr(), xs, _ptr(residual), rs,
                                        self.weight.data_ptr(), seed, call, None if plain else h.data_ptr(),
                                        None if self.fp8 else y, y if self.fp8 else None, _ptr(self._scale),
                                        _ptr(self._rstd), _stream(stream, self.device)))
        if self.fp8:
            return self._y, self._scale, h
        self._saved = (h, xs if plain else self.cols, seed, call, residual is not None)
        return self._y, h

    def backward(self, dy, dh=None, stream=None):
        """(dx, dresidual, dweight) after a forward call, from the gradients of y and of h (dh; None: zero). dresidual
        is None where the forward had no residual, and dx itself without dropout."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this norm first (and no 8-bit output)")
        h, hs, seed, call, residual = self._saved
        shape = (self.rows, self.cols)
        pdy = _full(dy, "dy", shape, self.dtype, self.device)
        pdh = None if dh is None else _full(dh, "dh", shape, self.dtype, self.device)
        if self._dx is None:
            self._dx = torch.empty(shape, dtype=self.dtype, device=self.device)
            self._dw = torch.empty(self.cols, dtype=torch.float32, device=self.device)
            self._ws = torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
        both = residual and self._drops
        if both and self._dres is None:
            self._dres = torch.empty(shape, dtype=self.dtype, device=self.device)
        check(lib().mdlstm_norm_backward(self.desc, self.rows, h.data_ptr(), hs, self._rstd.data_ptr(),
                                         self.weight.data_ptr(), pdy, pdh, seed, call,
                                         self._dx.data_ptr(), self._dres.data_ptr() if both else None,
                                         self._dw.data_ptr(), self._ws.data_ptr(), self._ws_bytes,
                                         _stream(stream, self.device)))
        return self._dx, (self._dres if both else self._dx) if residual else None, self._dw


def dropout(x, p: float, seed: int, call: int = 0, residual=None, out=None, stream=None) -> torch.Tensor:
    """residual + dropout(x) (residual None: dropout(x)) with a mask that is never stored: it follows from seed, call
    and an element's place in row-major order alone, so the gradient is the same call on the gradient of the result.
    p is taken to the nearest 2^-16; kept elements are scaled so that the expectation stays. x and residual:
    contiguous, or two-dimensional with contiguous rows. out: contiguous; may be x or residual."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("x must be a device tensor")
    shape, dt, dev = x.shape, x.dtype, x.device
    rows, cols = shape if len(shape) == 2 else (1, x.numel())

    def stride(t, name):
        if t.is_contiguous():
            return cols
        if len(shape) != 2:
            raise ValueError(f"{name} must be contiguous or two-dimensional")
        return _rows(t, name, shape, dt, dev)

    xs, rs, pres = stride(x, "x"), 0, None
    if residual is not None:
        _matches(residual, "residual", shape, dt, dev)
        rs, pres = stride(residual, "residual"), residual.data_ptr()
    if out is None:
        out = torch.empty(shape, dtype=dt, device=dev)
    check(lib().mdlstm_dropout(dtype_code(dt), rows, cols, x.data_ptr(), xs, p, _u64(seed, "seed"), _u64(call, "call"),
                               pres, rs, _full(out, "out", shape, dt, dev), _stream(stream, dev)))
    return out
