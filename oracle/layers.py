"""The gated recurrence, the group norm and the vocabulary's loss in float64 NumPy, from their definitions (see
include/mdlstm.h)."""
import numpy as np


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def gates(z, x, gate):
    """f and u of the recurrence h_t = f h_(t-1) + u."""
    z, x = np.asarray(z, np.float64), np.asarray(x, np.float64)
    return (_sigmoid(z), _sigmoid(-z) * x) if gate == "sigmoid" else (z, x)


def recurrence_forward(z, x, lengths, gate, state=None):
    """(h [T, C], final states [n, C])."""
    f, u = gates(z, x, gate)
    h = np.zeros_like(f)
    final = np.zeros((len(lengths), f.shape[1])) if state is None else np.array(state, np.float64)
    t = 0
    for i, n in enumerate(lengths):
        for _ in range(int(n)):
            final[i] = f[t] * final[i] + u[t]
            h[t] = final[i]
            t += 1
    return h, final


def recurrence_backward(z, x, lengths, gate, dh, state=None, dfinal=None):
    """(dz, dx, dstate) of sum(h * dh) + sum(final * dfinal)."""
    f, _ = gates(z, x, gate)
    h, _ = recurrence_forward(z, x, lengths, gate, state)
    x, dh = np.asarray(x, np.float64), np.asarray(dh, np.float64)
    dz, dx = np.zeros_like(f), np.zeros_like(f)
    adj = np.zeros((len(lengths), f.shape[1])) if dfinal is None else np.array(dfinal, np.float64)
    t0 = 0
    for i, n in enumerate(lengths):
        for t in range(t0 + int(n) - 1, t0 - 1, -1):
            before = h[t - 1] if t > t0 else (np.zeros(f.shape[1]) if state is None else np.asarray(state[i], np.float64))
            g = dh[t] + adj[i]
            if gate == "sigmoid":
                rest = _sigmoid(-np.asarray(z[t], np.float64))
                dz[t], dx[t] = g * (before - x[t]) * f[t] * rest, g * rest
            else:
                dz[t], dx[t] = g * before, g
            adj[i] = f[t] * g
        t0 += int(n)
    return dz, dx, adj


def _activation(u, act):
    """act(u) and its derivative."""
    if act == "silu":
        s = _sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "relu":
        return np.maximum(u, 0), (u > 0).astype(np.float64)
    return u, np.ones_like(u)


def group_norm(x, lengths, w, b, groups, eps, act, dy=None):
    """y, or with dy (dx, dw, db)."""
    x, w, b = (np.asarray(v, np.float64) for v in (x, w, b))
    C = x.shape[1]
    out, dw, db = np.zeros_like(x), np.zeros(C), np.zeros(C)
    t = 0
    for n in lengths:
        at = slice(t, t + int(n))
        t += int(n)
        if n == 0:
            continue
        v = x[at].reshape(-1, groups, C // groups)
        mean = v.mean(axis=(0, 2), keepdims=True)
        dev = np.sqrt(((v - mean) ** 2).mean(axis=(0, 2), keepdims=True) + eps)
        c = ((v - mean) / dev).reshape(-1, C)
        y, slope = _activation(c * w + b, act)
        if dy is None:
            out[at] = y
            continue
        e = np.asarray(dy[at], np.float64) * slope
        dw += (e * c).sum(0)
        db += e.sum(0)
        g, cg = (e * w).reshape(-1, groups, C // groups), c.reshape(-1, groups, C // groups)
        g = (g - g.mean(axis=(0, 2), keepdims=True) - cg * (g * cg).mean(axis=(0, 2), keepdims=True)) / dev
        out[at] = g.reshape(-1, C)
    return out if dy is None else (out, dw, db)


def vocabulary_loss(x, w, targets, dloss=None):
    """losses [T], or with dloss (dx, dw). A target outside the vocabulary: loss and gradients 0."""
    x, w, targets = np.asarray(x, np.float64), np.asarray(w, np.float64), np.asarray(targets)
    ok = (targets >= 0) & (targets < len(w))
    x = np.where(ok[:, None], x, 0.0)
    logits = x @ w.T
    top = logits.max(axis=1, keepdims=True)
    lse = np.log(np.exp(logits - top).sum(1)) + top[:, 0]
    at = np.where(ok, targets, 0)
    if dloss is None:
        return np.where(ok, lse - logits[np.arange(len(x)), at], 0.0)
    g = np.exp(logits - lse[:, None])
    g[np.arange(len(x)), at] -= 1.0
    g *= np.where(ok, np.asarray(dloss, np.float64), 0.0)[:, None]
    return g @ w, g.T @ x
