"""Sequence operators in float64 NumPy, from their definitions (see include/mdlstm.h).

attention_*: linear attention with a decay for each head, token by token.
norm_*: root-mean-square norm of a residual sum. dropout_scale: what dropout
multiplies each element by (0 or the scale).
"""
import math

import numpy as np


def _spread(x, heads):
    return np.repeat(np.asarray(x, np.float64), heads // x.shape[1], axis=1)


def attention_forward(q, k, v, lengths, rates, scale, state=None):
    """q [T, heads, dk], k [T, kv, dk], v [T, kv, dv] -> (o [T, heads, dv], final states [n, heads, dk, dv])."""
    heads = q.shape[1]
    q, k, v = np.asarray(q, np.float64), _spread(k, heads), _spread(v, heads)
    g = np.exp(-np.asarray(rates, np.float64))[:, None, None]
    o = np.zeros((q.shape[0], heads, v.shape[2]))
    final = np.zeros((len(lengths), heads, q.shape[2], v.shape[2]))
    t = 0
    for i, n in enumerate(lengths):
        S = np.zeros(final.shape[1:]) if state is None else np.asarray(state[i], np.float64)
        for _ in range(int(n)):
            S = g * S + k[t, :, :, None] * v[t, :, None, :]
            o[t] = scale * np.einsum("hi,hij->hj", q[t], S)
            t += 1
        final[i] = S
    return o, final


def attention_backward(q, k, v, lengths, rates, scale, do, state=None, dfinal=None):
    """(dq, dk, dv, dstate) of sum(o * do) + sum(final * dfinal)."""
    heads, kv = q.shape[1], k.shape[1]
    q, k, v, do = np.asarray(q, np.float64), _spread(k, heads), _spread(v, heads), np.asarray(do, np.float64)
    g = np.exp(-np.asarray(rates, np.float64))[:, None, None]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    dstate = np.zeros((len(lengths), heads, q.shape[2], v.shape[2]))
    t0 = 0
    for i, n in enumerate(lengths):
        n = int(n)
        S = np.zeros(dstate.shape[1:]) if state is None else np.asarray(state[i], np.float64)
        for t in range(t0, t0 + n):
            S = g * S + k[t, :, :, None] * v[t, :, None, :]
            dq[t] = scale * np.einsum("hij,hj->hi", S, do[t])
        G = np.zeros(dstate.shape[1:]) if dfinal is None else np.asarray(dfinal[i], np.float64)
        for t in range(t0 + n - 1, t0 - 1, -1):  # G: gradient of the state after token t
            G = G + scale * q[t, :, :, None] * do[t, :, None, :]
            dk[t] = np.einsum("hij,hj->hi", G, v[t])
            dv[t] = np.einsum("hij,hi->hj", G, k[t])
            G = g * G
        dstate[i] = G
        t0 += n
    shared = lambda x: x.reshape(x.shape[0], kv, heads // kv, x.shape[2]).sum(2)  # noqa: E731
    return dq, shared(dk), shared(dv), dstate


def attention_step(q, k, v, state, rates, slots, scale):
    """(o, states after): row i advances state slots[i]; a slot outside the states is an idle row."""
    heads = q.shape[1]
    q, k, v = np.asarray(q, np.float64), _spread(k, heads), _spread(v, heads)
    state = np.array(state, np.float64)
    g = np.exp(-np.asarray(rates, np.float64))[:, None, None]
    o = np.zeros((q.shape[0], heads, v.shape[2]))
    for i, s in enumerate(slots):
        if 0 <= s < state.shape[0]:
            state[s] = g * state[s] + k[i, :, :, None] * v[i, :, None, :]
            o[i] = scale * np.einsum("hi,hij->hj", q[i], state[s])
    return o, state


def philox(block, call, seed):
    """The four 32-bit words of Philox 4x32-10 with counter (block, call) and key seed, in Python integers."""
    low = 0xFFFFFFFF
    c = [block & low, block >> 32, call & low, call >> 32]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        p, r = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(r >> 32) ^ c[1] ^ k[0], r & low, (p >> 32) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def dropout_scale(n, p, seed, call):
    """[n] factors of the elements in row-major order."""
    t = round(p * 65536)
    if t == 0:
        return np.ones(n)
    if t == 65536:
        return np.zeros(n)
    u = [h for b in range(-(-n // 8)) for w in philox(b, call, seed) for h in (w & 0xFFFF, w >> 16)][:n]
    return np.where(np.asarray(u) >= t, 65536.0 / (65536 - t), 0.0)


def norm_forward(x, w, eps, residual=None, factor=None):
    """(y, h, rstd); factor: dropout_scale of the elements, in x's shape."""
    h = np.asarray(x, np.float64)
    if factor is not None:
        h = h * factor
    if residual is not None:
        h = h + np.asarray(residual, np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * np.asarray(w, np.float64), h, rstd


def norm_backward(h, w, eps, dy, dh=None, factor=None):
    """(dx, dresidual, dw) for the sum h."""
    h, w, dy = (np.asarray(a, np.float64) for a in (h, w, dy))
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    c, g = h * rstd, dy * w
    dres = rstd * (g - c * (g * c).mean(1, keepdims=True))
    if dh is not None:
        dres = dres + np.asarray(dh, np.float64)
    return dres if factor is None else dres * factor, dres, (dy * c).sum(0)


def unit_roundoff(dtype: str) -> float:
    """Largest relative error of one rounding to the storage type."""
    return math.ldexp(1.0, -8 if dtype == "bf16" else -24)
