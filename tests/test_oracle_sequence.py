"""Pins of the sequence oracle (oracle/sequence.py): hand-worked values, the
closed sum, gradients against central differences, a published Philox vector."""
import numpy as np

from oracle import sequence as os_


def _case(seed=0, heads=4, kv=2, dk=3, dv=5, lengths=(4, 0, 1, 6)):
    rng = np.random.default_rng(seed)
    T = sum(lengths)
    return (rng.standard_normal((T, heads, dk)), rng.standard_normal((T, kv, dk)), rng.standard_normal((T, kv, dv)),
            np.array(lengths), rng.uniform(0, 0.5, heads), rng.standard_normal((len(lengths), heads, dk, dv)), rng)


def test_attention_by_hand():
    """Two tokens of one head, dims 1, decay 1/2: o = 2 q (k v), then q (k v / 2 + k v)."""
    q, k, v = (np.array(a, float).reshape(2, 1, 1) for a in ([1, 3], [2, 1], [5, 7]))
    o, final = os_.attention_forward(q, k, v, [2], [np.log(2.0)], 2.0)
    assert np.allclose(o.ravel(), [2 * 10, 2 * 3 * (5 + 7)]) and np.allclose(final.ravel(), [12])
    # two sequences of one token: the state restarts
    o, _ = os_.attention_forward(q, k, v, [1, 1], [np.log(2.0)], 2.0)
    assert np.allclose(o.ravel(), [20, 2 * 3 * 7])


def test_attention_is_the_closed_sum():
    q, k, v, n, a, S0, _ = _case()
    o, final = os_.attention_forward(q, k, v, n, a, 0.7, S0)
    t0 = 0
    for i, m in enumerate(n):
        for h in range(4):
            j = h // 2
            for t in range(m):
                want = np.exp(-a[h] * (t + 1)) * q[t0 + t, h] @ S0[i, h]
                for s in range(t + 1):
                    want = want + np.exp(-a[h] * (t - s)) * (q[t0 + t, h] @ k[t0 + s, j]) * v[t0 + s, j]
                assert np.allclose(o[t0 + t, h], 0.7 * want)
        if m == 0:
            assert np.array_equal(final[i], S0[i])
        t0 += m


def test_attention_gradients_by_differences():
    q, k, v, n, a, S0, rng = _case(1)
    do, df = rng.standard_normal((q.shape[0], 4, 5)), rng.standard_normal(S0.shape)

    def loss(q, k, v, S0):
        o, f = os_.attention_forward(q, k, v, n, a, 0.7, S0)
        return (o * do).sum() + (f * df).sum()

    grads = os_.attention_backward(q, k, v, n, a, 0.7, do, S0, df)
    args = [q, k, v, S0]
    for i, g in enumerate(grads):
        d = rng.standard_normal(g.shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-4 * d, args[i] - 1e-4 * d
        num = (loss(*up) - loss(*down)) / 2e-4
        assert abs(num - (g * d).sum()) < 1e-6 * max(1.0, abs(num)), i


def test_step_continues_a_sequence():
    q, k, v, _, a, S0, _ = _case(2, lengths=(7,))
    o, final = os_.attention_forward(q, k, v, [7], a, 0.3, S0)
    st = S0
    for t in range(7):
        ot, st = os_.attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], st, a, [0], 0.3)
        assert np.allclose(ot[0], o[t])
    assert np.allclose(st, final)
    ot, same = os_.attention_step(q[:1], k[:1], v[:1], st, a, [-1], 0.3)
    assert not ot.any() and np.array_equal(same, st)


def test_philox_published_vectors():
    """Known answers of the Philox 4x32-10 paper's library: zero counter and key, all ones, digits of pi."""
    assert os_.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = (1 << 64) - 1
    assert os_.philox(ones, ones, ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert os_.philox(0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_the_share_and_the_mean():
    f = os_.dropout_scale(40000, 0.3, 17, 5)
    assert abs((f == 0).mean() - 0.3) < 5 * np.sqrt(0.21 / 40000)
    assert abs(f.mean() - 1) < 5 * np.sqrt(0.3 / 0.7 / 40000)
    assert not np.array_equal(f, os_.dropout_scale(40000, 0.3, 17, 6))
    assert not os_.dropout_scale(9, 1.0, 1, 1).any() and os_.dropout_scale(9, 0.0, 1, 1).all()


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(3)
    x, r, w = rng.standard_normal((5, 7)), rng.standard_normal((5, 7)), rng.standard_normal(7)
    dy, dh = rng.standard_normal((5, 7)), rng.standard_normal((5, 7))
    f = os_.dropout_scale(35, 0.4, 3, 2).reshape(5, 7)

    def loss(x, r, w):
        y, h, _ = os_.norm_forward(x, w, 1e-3, r, f)
        return (y * dy).sum() + (h * dh).sum()

    _, h, _ = os_.norm_forward(x, w, 1e-3, r, f)
    grads, args = os_.norm_backward(h, w, 1e-3, dy, dh, f), [x, r, w]
    for i, g in enumerate(grads):
        d = rng.standard_normal(g.shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * d, args[i] - 1e-5 * d
        num = (loss(*up) - loss(*down)) / 2e-5
        assert abs(num - (g * d).sum()) < 1e-6 * max(1.0, abs(num)), i
