"""The oracle of the gated recurrence, the group norm and the vocabulary's loss against torch's float64 autograd of the
same formulas, written apart."""
import numpy as np
import pytest

from oracle import layers as orc

torch = pytest.importorskip("torch")


def _t(a):
    return torch.from_numpy(np.array(a)).requires_grad_()


@pytest.mark.parametrize("gate", ["sigmoid", None])
def test_recurrence(gate):
    rng = np.random.default_rng(1)
    lengths, C = [3, 0, 5, 1], 4
    z, x, dh, state, df = (rng.standard_normal(s) for s in ((9, C), (9, C), (9, C), (4, C), (4, C)))
    tz, tx, ts = _t(z), _t(x), _t(state)
    out, finals, t = [], [], 0
    for i, n in enumerate(lengths):
        h = ts[i]
        for _ in range(n):
            f = torch.sigmoid(tz[t]) if gate else tz[t]
            h = f * h + ((1 - f) * tx[t] if gate else tx[t])
            out.append(h)
            t += 1
        finals.append(h)
    out, finals = torch.stack(out), torch.stack(finals)
    (out * torch.from_numpy(dh)).sum().add((finals * torch.from_numpy(df)).sum()).backward()
    h, final = orc.recurrence_forward(z, x, lengths, gate, state)
    assert np.allclose(h, out.detach()) and np.allclose(final, finals.detach())
    for got, want in zip(orc.recurrence_backward(z, x, lengths, gate, dh, state, df), (tz.grad, tx.grad, ts.grad)):
        assert np.allclose(got, want)


@pytest.mark.parametrize("act", [None, "relu", "silu"])
def test_group_norm(act):
    rng = np.random.default_rng(2)
    lengths, C, G = [4, 0, 7], 6, 3
    x, dy, w, b = (rng.standard_normal(s) for s in ((11, C), (11, C), C, C))
    tx, tw, tb = _t(x), _t(w), _t(b)
    parts = []
    for v in torch.split(tx, lengths):
        if len(v):
            y = torch.nn.functional.group_norm(v.t()[None], G, tw, tb, 1e-5)[0].t()
            parts.append(torch.relu(y) if act == "relu" else torch.nn.functional.silu(y) if act else y)
    y = torch.cat(parts)
    (y * torch.from_numpy(dy)).sum().backward()
    assert np.allclose(orc.group_norm(x, lengths, w, b, G, 1e-5, act), y.detach())
    for got, want in zip(orc.group_norm(x, lengths, w, b, G, 1e-5, act, dy), (tx.grad, tw.grad, tb.grad)):
        assert np.allclose(got, want)


def test_vocabulary_loss():
    rng = np.random.default_rng(3)
    x, w, dl = rng.standard_normal((7, 5)), rng.standard_normal((11, 5)), rng.standard_normal(7)
    t = np.array([0, 10, 3, -1, 3, 11, 7])
    tx, tw = _t(x), _t(w)
    losses = torch.nn.functional.cross_entropy(tx @ tw.t(), torch.from_numpy(np.where((t >= 0) & (t < 11), t, -100)), reduction="none")
    (losses * torch.from_numpy(dl)).sum().backward()
    assert np.allclose(orc.vocabulary_loss(x, w, t), losses.detach())
    for got, want in zip(orc.vocabulary_loss(x, w, t, dl), (tx.grad, tw.grad)):
        assert np.allclose(got, want)
