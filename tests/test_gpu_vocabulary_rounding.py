"""How far rounding takes the gradients of the softmax cross entropy over a vocabulary in bf16, against the float64
oracle (oracle/layers.py), number by number.

Tolerances. A result is a sum in fp32, rounded to bf16 once: 2^-8 of itself. The sum's terms are products of a bf16
number and of q (c q in dW) in two bf16 pieces, 2^-16 of each term; sums of up to 2^12 terms go through fewer than 256
fp32 additions one after another (32 terms a matrix instruction, parts of the sum, pieces of the vocabulary), 2^-24 each:
2^-16. So a number is at most 2^-8 of itself and 2^-15 of the sum of its terms' magnitudes off. Logits of 128
products are off by at most 40 roundings of 2^-24 of the sum of magnitudes, and a logit's error moves its own q by as much:
of rows of W that share a part only what they do not share, as the q of a row add up to 1 whatever the logits are."""
import numpy as np
import pytest

from oracle import layers as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16().cuda()


def _gradients(x, w, t, dl):
    from paper_1902_11208_amd import sequence

    op = sequence.VocabularyLoss(w, x.shape[0])
    op.forward(x, torch.from_numpy(t).cuda())
    return [_np(g) for g in op.backward(torch.from_numpy(dl.astype(np.float32)).cuda())]


def _terms(x, w, t, dl):
    """|dl_v| of every row, [rows][vocab]."""
    l = x @ w.T
    g = np.exp(l - l.max(1, keepdims=True))
    g /= g.sum(1, keepdims=True)
    g[np.arange(len(x)), t] -= 1.0
    return np.abs(g) * dl[:, None]


def _bounds(x, w, t, dl, shared):
    """The tolerances of dx and dw beside 2^-8 of themselves."""
    g = _terms(x, w, t, dl)
    logits = 40 * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T).max()
    own = np.abs(w - shared)
    return 2.0 ** -15 * (g @ np.abs(w)) + 2 * logits * (g @ own), 2.0 ** -15 * (g.T @ np.abs(x)) + 2 * logits * (g.T @ np.abs(x))


@pytest.mark.parametrize("common", [0.0, 1.0, 3.0, 10.0])
@pytest.mark.parametrize("rows,vocab", [(60, 2000), (700, 3000)])
def test_rows_of_w_with_a_common_part(rows, vocab, common):
    """What W's rows share falls out of dx, as the softmax's gradient adds up to 0 over the vocabulary."""
    rng = np.random.default_rng(rows)
    shared = common * np.sign(rng.standard_normal(128))  # exact in bf16
    w = _bf16(shared + 0.18 * rng.standard_normal((vocab, 128)))
    x = _bf16(0.3 * rng.standard_normal((rows, 128)))
    t, dl = rng.integers(0, vocab, rows), rng.uniform(0.5, 1.5, rows).astype(np.float32).astype(np.float64)
    nx, nw = _np(x), _np(w)
    want = orc.vocabulary_loss(nx, nw, t, dl)
    for name, got, ref, more in zip(("dx", "dw"), _gradients(x, w, t, dl), want, _bounds(nx, nw, t, dl, shared)):
        off = np.abs(got - ref) / (2.0 ** -8 * np.abs(ref) + more)
        assert off.max() <= 1, (name, off.max(), np.argmax(off))


@pytest.mark.parametrize("rows,dim,vocab", [(1000, 64, 150), (3000, 64, 700), (2000, 100, 9000), (500, 64, 70000), (300, 128, 66000)])
@pytest.mark.parametrize("dloss", [1.0019, 1.0058, 1.5 / 4096])
def test_one_gradient_for_all_losses(rows, dim, vocab, dloss):
    """All losses with one gradient and no target likely: c is one number in all rows, and were it rounded, all of dW
    would be off the same way. Rounding results leaves them without bias: the part of the error along dW is a mean of
    independent errors of at most 2^-8 each, here of the thousands of numbers of the targets' rows: within five times
    2^-8 / sqrt(their number), and 2^-15. The rows of dW of a vocabulary in one piece and in several, stored by their product
    and as planes."""
    rng = np.random.default_rng(vocab)
    w, x = _bf16(0.05 * rng.standard_normal((vocab, dim))), _bf16(1 + 0.5 * rng.standard_normal((rows, dim)))
    hot = np.r_[rng.integers(0, vocab, 40), vocab - 1]  # also in the last piece
    t = rng.choice(hot, rows)
    dl = np.full(rows, np.float32(dloss), np.float64)
    nx, nw = _np(x), _np(w)
    _, got = _gradients(x, w, t, dl)
    _, want = orc.vocabulary_loss(nx, nw, t, dl)
    at = np.unique(t)
    e, ref = got[at] - want[at], want[at]
    assert abs((e * ref).sum() / (ref * ref).sum()) <= 5 * 2.0 ** -8 / np.sqrt(ref.size) + 2.0 ** -15
    _, more = _bounds(nx, nw, t, dl, 0.0)
    off = np.abs(got - want) / (2.0 ** -8 * np.abs(want) + more + 1e-40)
    assert off.max() <= 1, off.max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(40, 300), (300, 2500), (1100, 20000)])
def test_logits_of_a_thousand(rows, vocab, dtype):
    """Logits that share 1000, all of them exact in fp32: multiples of 1/64 below 2^11. A loss is a difference from them: its
    exponents (of terms that count: at most 2^5 below the largest) are rounded at 2^-20 and each sum at 2^-24 of itself some
    twenty times, 2^-19 of 1 + loss in all. The q of a row add up to 1 as far, and their product with a column of ones (48
    additions of 2^-24, pieces of 2^-24, or of 2^-16 in bf16) is 0 but for as much: 2^-18 of c, 2^-15 in bf16."""
    from paper_1902_11208_amd import sequence

    rng = np.random.default_rng(rows)
    eighths = lambda *s: np.clip(np.rint(8 * rng.standard_normal(s)), -24, 24) / 8  # noqa: E731
    x, w = eighths(rows, 24), eighths(vocab, 24)
    x[:, 8:], x[:, 0], w[:, 0] = 0, 1000, 1
    t, dl = rng.integers(0, vocab, rows), rng.uniform(0.5, 1.5, rows).astype(np.float32).astype(np.float64)
    op = sequence.VocabularyLoss(torch.from_numpy(w).to(dtype).cuda(), rows)
    losses = _np(op.forward(torch.from_numpy(x).to(dtype).cuda(), torch.from_numpy(t).cuda()))
    want = orc.vocabulary_loss(x, w, t)
    off = np.abs(losses - want) / (2.0 ** -19 * (1 + want))
    assert off.max() <= 1, off.max()
    dx, _ = op.backward(torch.from_numpy(dl.astype(np.float32)).cuda())
    off = np.abs(_np(dx)[:, 0]) / dl
    assert off.max() <= (2.0 ** -18 if dtype == torch.float32 else 2.0 ** -15), off.max()
