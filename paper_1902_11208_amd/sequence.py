"""Layers along the packed frames of the examples (or any packed tokens):
linear attention with a decay for each head, a gated linear recurrence, the
single-token steps of both, root-mean-square norm of a residual sum, dropout, a
norm over groups of channels with an activation, and the softmax cross entropy over
a vocabulary.

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

from ._lib import AttentionDesc, GroupNormDesc, NormDesc, RecurrenceDesc, VocabularyDesc, lib
from .api import check_tensor, dtype_code

try:
    from . import _binding
except ImportError as e:
    raise RuntimeError("the native binding is missing: build it with `python -m paper_1902_11208_amd.build`") from e

FP8 = torch.float8_e4m3fn
GATES = {None: 0, "sigmoid": 1}
ACTIVATIONS = {None: 0, "relu": 1, "silu": 2}


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


class _PackedLayer:
    """Sequences of given lengths, packed: where they start, and the order in which they are started."""

    def __init__(self, lengths, channels: int, dtype, device):
        n = np.asarray(lengths, np.int64).reshape(-1)
        if n.size and n.min() < 0:
            raise ValueError("a sequence has a negative length")
        self.n, self.tokens, self.longest = int(n.size), int(n.sum()), int(n.max()) if n.size else 0
        self.channels, self.dtype = int(channels), dtype
        self._lengths, self._device = n, torch.device(device)

    def _bytes_of(self, call, *args) -> int:
        nbytes = int(call(*args))
        if not nbytes:
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        return nbytes

    def _upload(self):
        n = self._lengths
        self.offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(self._device)
        # longest first, so that no long sequence starts when the others are done
        self.order = torch.from_numpy(np.argsort(-n, kind="stable").astype(np.int32)).to(self._device)
        self.device = self.offsets.device
        self._ws, self._saved = [None, None], None

    def _workspace(self, backward: int, stream) -> torch.Tensor:
        if self._ws[backward] is None:
            self._ws[backward] = _empty(self._bytes[backward], torch.uint8, self.device, stream)
        return self._ws[backward]


class GatedRecurrence(_PackedLayer):
    """Gated linear recurrence over packed sequences, for each channel

        h_t = f_t h_(t-1) + u_t        gate "sigmoid": f = sigmoid(z), u = (1 - f) x        gate None: f = z, u = x

    the state in fp32 restarting at every sequence's edge. lengths: tokens of each sequence (host); zero is allowed.
    dtype: storage of z, x, h and their gradients; sums and states are fp32, and outputs are rounded once.

    States that a call returned may be given back to the object, to go through sequences piece by piece: a call
    writes to a buffer that neither its arguments nor the forward call it belongs to use. Its other outputs must not be
    its inputs.
    """

    def __init__(self, lengths, channels: int, dtype=torch.bfloat16, gate: str = "sigmoid", device="cuda"):
        if gate not in GATES:
            raise ValueError(f"gate {gate!r} is not None or 'sigmoid'")
        super().__init__(lengths, channels, dtype, device)
        desc = RecurrenceDesc(self.channels, dtype_code(dtype), GATES[gate])
        self._bytes = [self._bytes_of(lib().mdlstm_recurrence_workspace_bytes, ctypes.byref(desc), self.n, self.tokens,
                                      self.longest, b) for b in (0, 1)]
        self._marks_bytes = self._bytes_of(lib().mdlstm_recurrence_marks_bytes, ctypes.byref(desc), self.tokens)
        self._upload()
        self._op = _binding.Recurrence(self.channels, desc.dtype, desc.gate, self.n, self.tokens, self.longest, self.offsets,
                                       self.order)
        self._h = self._marks = self._grads = None
        self._finals, self._dstates = [], []

    def _spare(self, buffers: list, stream, *used) -> torch.Tensor:
        """The first of the buffers of states that none of `used` lies in."""
        for b in buffers:
            if all(_apart(b, u) for u in used):
                return b
        buffers.append(_empty((self.n, self.channels), torch.float32, self.device, stream))
        return buffers[-1]

    def forward(self, z, x, state=None, final_state: bool = False, stream=None):
        """h [tokens, channels]; with final_state also the states the sequences leave [n, channels]. state: the states
        they start from (None: zero). z and x: [tokens, channels], contiguous along their rows (views of one
        projection's output, say)."""
        if self._h is None:
            self._h = _empty((self.tokens, self.channels), self.dtype, self.device, stream)
            self._marks = _empty(self._marks_bytes // 4, torch.float32, self.device, stream)
        final = self._spare(self._finals, stream, state) if final_state else None
        self._op.forward(z, x, state, self._h, final, self._marks, self._workspace(0, stream), _stream(stream))
        self._saved = (z, x, state)
        return (self._h, final) if final_state else self._h

    def backward(self, dh, dstate=None, stream=None):
        """(dz, dx) after a forward call, from the gradient of h (and of the final states, dstate); where the forward
        was given states, (dz, dx, gradient of those)."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this layer first")
        z, x, state = self._saved
        if self._grads is None:
            self._grads = tuple(_empty((self.tokens, self.channels), self.dtype, self.device, stream) for _ in range(2))
        out = None if state is None else self._spare(self._dstates, stream, state, dstate)
        self._op.backward(z, x, state, self._marks, dh, dstate, *self._grads, out, self._workspace(1, stream), _stream(stream))
        return self._grads if state is None else self._grads + (out,)


def gated_recurrence_step(z, x, state, slots=None, gate: str = "sigmoid", out=None, stream=None) -> torch.Tensor:
    """One token for each of n sequences: z and x [n, channels] advance the fp32 states [slots, channels] in place and
    give h [n, channels]. slots: int32 [n] device tensor, the state of each row (None: row i has state i); a slot
    outside the states marks an idle row, whose h is zero. No two rows may name the same slot."""
    if gate not in GATES:
        raise ValueError(f"gate {gate!r} is not None or 'sigmoid'")
    return _binding.recurrence_step(z, x, state, slots, GATES[gate], out, _stream(stream))


class GroupNorm(_PackedLayer):
    """Norm over groups of channels with an activation, channels last, over packed sequences:

        y = act((x - mean) / sqrt(var + eps) * weight + bias)

    mean and var over the tokens of a sequence (pixels of an image) and the channels of a group, channels / groups
    neighbouring ones. weight, bias: [channels] fp32 device tensors. activation: None, "relu" or "silu". dtype: storage
    of x, y and their gradients; sums are fp32.
    """

    def __init__(self, lengths, weight: torch.Tensor, bias: torch.Tensor, groups: int, dtype=torch.bfloat16, eps: float = 1e-5,
                 activation: str = None):
        if not isinstance(weight, torch.Tensor) or weight.dim() != 1:
            raise ValueError("weight must be a [channels] tensor")
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation {activation!r} is not None, 'relu' or 'silu'")
        super().__init__(lengths, weight.numel(), dtype, weight.device)
        check_tensor(weight, "weight", (self.channels,), torch.float32)
        check_tensor(bias, "bias", (self.channels,), torch.float32, weight.device)
        self.weight, self.bias, self.groups = weight, bias, int(groups)
        desc = GroupNormDesc(self.channels, self.groups, dtype_code(dtype), ACTIVATIONS[activation], float(eps))
        self._bytes = [self._bytes_of(lib().mdlstm_group_norm_workspace_bytes, ctypes.byref(desc), self.n, self.tokens,
                                      self.longest, b) for b in (0, 1)]
        self._upload()
        self._op = _binding.GroupNorm(self.channels, self.groups, desc.dtype, desc.activation, desc.eps, self.n, self.tokens,
                                      self.longest, self.offsets, self.order, weight, bias)
        self._y = self._stats = self._grads = None

    def forward(self, x, stream=None) -> torch.Tensor:
        """y [tokens, channels] of x [tokens, channels], contiguous along its rows."""
        if self._y is None:
            self._y = _empty((self.tokens, self.channels), self.dtype, self.device, stream)
            self._stats = [_empty((self.n, self.groups), torch.float32, self.device, stream) for _ in range(2)]
        self._op.forward(x, self._y, *self._stats, self._workspace(0, stream), _stream(stream))
        self._saved = x
        return self._y

    def backward(self, dy, stream=None):
        """(dx, dweight, dbias) after a forward call, from the gradient of y. Weight and bias have to be as they were in
        the forward call."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this norm first")
        if self._grads is None:
            self._grads = (_empty((self.tokens, self.channels), self.dtype, self.device, stream),
                           _empty(self.channels, torch.float32, self.device, stream),
                           _empty(self.channels, torch.float32, self.device, stream))
        self._op.backward(self._saved, *self._stats, dy, *self._grads, self._workspace(1, stream), _stream(stream))
        return self._grads


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


class VocabularyLoss:
    """Softmax cross entropy of `rows` rows over a vocabulary, without stored logits:

        loss_i = log(sum_v exp(x_i . weight_v)) - x_i . weight_target_i

    weight: [vocab, dim] device tensor, float32 or bfloat16, which x and the gradients share. A row whose target lies
    outside [0, vocab) (-1, say) has loss 0 and takes no part in the gradients, whatever it holds. Sums are fp32, and
    gradients are rounded to bfloat16 once.
    """

    def __init__(self, weight: torch.Tensor, rows: int):
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise ValueError("weight must be a [vocab, dim] tensor")
        desc = VocabularyDesc(weight.shape[1], weight.shape[0], dtype_code(weight.dtype))
        check_tensor(weight, "weight", weight.shape, weight.dtype)
        self.weight, self.rows, self.vocab, self.dim = weight, int(rows), weight.shape[0], weight.shape[1]
        self.dtype, self.device = weight.dtype, weight.device
        self._bytes = [int(lib().mdlstm_vocabulary_workspace_bytes(ctypes.byref(desc), self.rows, b)) for b in (0, 1)]
        if not all(self._bytes):
            raise ValueError(lib().mdlstm_last_error().decode(errors="replace"))
        self._op = _binding.Vocabulary(self.dim, self.vocab, desc.dtype, self.rows, weight)
        self._losses = self._stats = self._grads = self._saved = None
        self._ws = [None, None]

    def _workspace(self, backward: int, stream) -> torch.Tensor:
        if self._ws[backward] is None:
            self._ws[backward] = _empty(self._bytes[backward], torch.uint8, self.device, stream)
        return self._ws[backward]

    def forward(self, x, targets, stream=None) -> torch.Tensor:
        """losses [rows] in fp32 of x [rows, dim], contiguous along its rows, and targets [rows] (int64)."""
        if self._losses is None:
            self._losses = _empty(self.rows, torch.float32, self.device, stream)
            self._stats = _empty((2, self.rows), torch.float32, self.device, stream)
        self._op.forward(x, targets, self._losses, self._stats, self._workspace(0, stream), _stream(stream))
        self._saved = (x, targets)
        return self._losses

    def backward(self, dlosses, stream=None):
        """(dx, dweight) in the storage type after a forward call, from the gradient of the losses [rows] (fp32). The
        weights have to be as they were in the forward call."""
        if self._saved is None:
            raise ValueError("backward needs a forward call on this loss first")
        if self._grads is None:
            self._grads = (_empty((self.rows, self.dim), self.dtype, self.device, stream),
                           _empty((self.vocab, self.dim), self.dtype, self.device, stream))
        self._op.backward(*self._saved, self._stats, dlosses, *self._grads, self._workspace(1, stream), _stream(stream))
        return self._grads


def dropout(x, p: float, seed: int, call: int = 0, residual=None, out=None, stream=None) -> torch.Tensor:
    """residual + dropout(x) (residual None: dropout(x)) with a mask that is never stored: it follows from seed, call
    and an element's place in row-major order alone, so the gradient is the same call on the gradient of the result.
    p is taken to the nearest 2^-16; kept elements are scaled so that the expectation stays. x and residual:
    contiguous, or two-dimensional with contiguous rows. out: contiguous; may be x or residual."""
    return _binding.dropout(x, p, _u64(seed, "seed"), _u64(call, "call"), residual, out, _stream(stream))
