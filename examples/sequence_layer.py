"""A sequence layer between an MDLSTM layer and the CTC loss, trained and then served column by column.

    images -> packed canvas -> MDLSTM layer -> frames (rows summed) -> dropout -> h
    h' = h + dropout(attention(norm(h)) Wo)       y = norm(h')       logits = y Wc + bc -> CTC

The canvas, the frames and the sequence layer all stay packed: no example is padded, and the attention's state
restarts at every example's edge. Its heads are the four scan directions. Serving then reads most of a line as a
prompt, keeps the state it leaves and advances it one column at a time; the last norm is also run with its 8-bit
output, whose product with the classes' weights is compared. The plain products are torch's.

    python examples/sequence_layer.py [--steps N] [--examples N]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1902_11208_amd import api, sequence  # noqa: E402
from synth import configs  # noqa: E402

DIRECTIONS = 4


class SequenceLayer:
    """norm, attention over the frames, projection, dropout and residual, norm, classes."""

    def __init__(self, lengths, width, classes, dropout, gen, device="cuda"):
        self.head_dim, T = width // DIRECTIONS, int(np.sum(lengths))
        new = lambda *s: torch.randn(s, generator=gen, device=device) * s[0] ** -0.5  # noqa: E731
        rates = torch.tensor([2.0 ** -(3 + 2 * h) for h in range(DIRECTIONS)], device=device)
        self.w = {"qkv": new(width, 3 * width), "o": new(width, width), "c": new(width, classes),
                  "bc": torch.zeros(classes, device=device), "n1": torch.ones(width, device=device),
                  "n2": torch.ones(width, device=device)}
        self.rates = rates
        self.n1 = sequence.ResidualNorm(self.w["n1"], T, dtype=torch.float32)
        self.n2 = sequence.ResidualNorm(self.w["n2"], T, dtype=torch.float32, dropout=dropout)
        self.attention = sequence.DecayAttention(lengths, DIRECTIONS, self.head_dim, self.head_dim, rates,
                                                 dtype=torch.float32)

    def split(self, qkv):
        return (t.unflatten(1, (DIRECTIONS, self.head_dim)) for t in qkv.chunk(3, 1))  # views: nothing is copied

    def forward(self, h, seed, call):
        y1, _ = self.n1.forward(h)
        self.q, self.k, self.v = self.split(y1 @ self.w["qkv"])
        self.y1, self.o = y1, self.attention.forward(self.q, self.k, self.v).flatten(1)
        self.y2, _ = self.n2.forward(self.o @ self.w["o"], h, seed=seed, call=call)
        return self.y2 @ self.w["c"] + self.w["bc"]

    def backward(self, dlogits):
        """Gradient of h, and of the weights."""
        du, dh, dn2 = self.n2.backward(dlogits @ self.w["c"].t())
        dq, dk, dv = self.attention.backward((du @ self.w["o"].t()).unflatten(1, (DIRECTIONS, self.head_dim)))
        dqkv = torch.cat([t.flatten(1) for t in (dq, dk, dv)], 1)
        dx, _, dn1 = self.n1.backward(dqkv @ self.w["qkv"].t(), dh)  # h is the norm's input and the residual
        return dx, {"qkv": self.y1.t() @ dqkv, "o": self.o.t() @ du, "c": self.y2.t() @ dlogits,
                    "bc": dlogits.sum(0), "n1": dn1, "n2": dn2}

    def serve(self, h, last):
        """Logits of the last `last` frames of one line h [frames, width], a column at a time after a prompt."""
        n, w, eps = h.shape[0] - last, self.w, 1e-6
        new = lambda weight, rows, **kw: sequence.ResidualNorm(weight, rows, dtype=torch.float32, eps=eps, **kw)  # noqa: E731
        prompt = sequence.DecayAttention([n], DIRECTIONS, self.head_dim, self.head_dim, self.rates, dtype=torch.float32)
        _, state = prompt.forward(*self.split(new(w["n1"], n).forward(h[:n])[0] @ w["qkv"]), final_state=True)
        n1, n2, n8 = new(w["n1"], 1), new(w["n2"], 1), new(w["n2"], 1, out="fp8")
        logits, logits8 = [], []
        for t in range(n, h.shape[0]):
            column = h[t:t + 1].contiguous()
            q, k, v = self.split(n1.forward(column)[0] @ w["qkv"])
            u = sequence.decay_attention_step(q, k, v, state, self.rates).flatten(1) @ w["o"]
            logits.append(n2.forward(u, column)[0] @ w["c"] + w["bc"])
            y8, scale, _ = n8.forward(u, column)
            logits8.append(y8.float() @ w["c"] * scale[:, None] + w["bc"])
        return torch.cat(logits), torch.cat(logits8)


def main(steps=30, examples=24, hidden=16, dropout=0.1, rate=0.05, seed=7):
    """(losses of the steps, error of the served logits, error with the 8-bit output)."""
    rng = np.random.default_rng(seed)
    wl = configs.custom_workload(97, np.full(examples, 16), rng.integers(20, 80, examples), 512, 1, hidden)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rects, canvas_h, mask = api.pack_layout(wl.heights, wl.widths, wl.canvas_w)
    x = api.pack_data([torch.from_numpy(e).cuda() for e in wl.examples()], rects, canvas_h, wl.canvas_w)
    wx, u, b = (torch.from_numpy(p).cuda() for p in wl.params())
    layer = api.MDLSTMLayer(wx, u, b, canvas_h, wl.canvas_w, rects, mask)
    labels = [wl.label(k, 12) for k in range(examples)]
    W, bias = (torch.from_numpy(p).cuda() for p in wl.head_params(12))
    head = api.Head(W, bias, rects, (canvas_h, wl.canvas_w), labels)  # its CTC loss; the classes come from the new layer
    seq = SequenceLayer(wl.widths, DIRECTIONS * hidden, 12, dropout, gen)
    # frame of every canvas cell, for the sum over an example's rows and its gradient
    frame = np.full((canvas_h, wl.canvas_w), -1, np.int64)
    off = np.concatenate([[0], np.cumsum(wl.widths)])
    for i, (y0, x0, h, w) in enumerate(rects):
        frame[y0:y0 + h, x0:x0 + w] = off[i] + np.arange(w)
    cells = torch.from_numpy(np.flatnonzero(frame.ravel() >= 0)).cuda()
    frame = torch.from_numpy(frame.ravel()).cuda()[cells]
    width, T = DIRECTIONS * hidden, int(off[-1])
    losses = []
    for step in range(steps):
        y = layer.forward(x).view(-1, width)
        frames = torch.zeros(T, width, device="cuda").index_add_(0, frame, y[cells])
        h = sequence.dropout(frames, dropout, seed, 2 * step)
        loss, dlogits = head.ctc(seq.forward(h, seed, 2 * step + 1))
        losses.append(float(loss.mean()))
        dh, grads = seq.backward(dlogits / examples)
        dy = torch.zeros(canvas_h * wl.canvas_w, width, device="cuda")
        dy[cells] = sequence.dropout(dh, dropout, seed, 2 * step)[frame]
        _, dwx, du, db = layer.backward(dy.view(canvas_h, wl.canvas_w, width))
        for p, g in [(layer.wx, dwx), (layer.u, du), (layer.b, db)] + [(seq.w[k], grads[k]) for k in grads]:
            p -= rate / max(1.0, float(g.norm())) * g
    # one line served: a prompt, then its last ten columns one by one, against the whole line at once
    line = sequence.DecayAttention([int(wl.widths[0])], DIRECTIONS, seq.head_dim, seq.head_dim, seq.rates, dtype=torch.float32)
    h = frames[:int(wl.widths[0])].contiguous()
    new = lambda name: sequence.ResidualNorm(seq.w[name], h.shape[0], dtype=torch.float32)  # noqa: E731
    o = line.forward(*seq.split(new("n1").forward(h)[0] @ seq.w["qkv"])).flatten(1)
    whole = (new("n2").forward(o @ seq.w["o"], h)[0] @ seq.w["c"] + seq.w["bc"])[-10:]
    served, served8 = seq.serve(h, 10)
    err = [float((s - whole).norm() / whole.norm()) for s in (served, served8)]
    return losses, err[0], err[1]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--examples", type=int, default=24)
    a = ap.parse_args()
    losses, err, err8 = main(a.steps, a.examples)
    print(f"CTC loss of an example: {losses[0]:.2f} -> {losses[-1]:.2f} in {len(losses)} steps")
    print(f"served column by column against the whole line: {err:.1e}; with the 8-bit norm: {err8:.1e}")
