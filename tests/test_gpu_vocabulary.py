"""GPU parity of the softmax cross entropy over a vocabulary against the float64
oracle (oracle/layers.py).

Tolerances, normwise L2 and max-norm relative error. fp32: 1e-5 as for the other
layers. bf16: losses are fp32 sums, 1e-5; in a gradient each factor q of a sum is
rounded to bf16 (at most 2^-9 relative each, all terms together at most 2^-9 of
the sum of magnitudes) and the result is rounded once (2^-9 relative, so 2^-8 of a
step at most): the sum of magnitudes is at most twice what the target's exact
share and the softmax's share leave where nothing cancels, so 4 * 2^-9 bounds both."""
import numpy as np
import pytest

from conftest import rel_err, rel_max
from oracle import layers as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = {"f32": 1e-5, "bf16": 4 * 2.0 ** -9}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _loss(*a):
    from paper_1902_11208_amd import sequence

    return sequence.VocabularyLoss(*a)


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _check(name, got, want, tol):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    e, m = rel_err(got, want), rel_max(got, want)
    assert e <= tol and m <= tol, (name, e, m)


def _rand(rng, *shape, dtype="f32", scale=1.0):
    return torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).to(DT[dtype]).cuda()


def _case(rng, rows, dim, vocab, dtype, odd=False):
    """x, weights, targets with every fourth row left out (where there are four), gradients of the losses."""
    x = _rand(rng, rows, dim + 3 * odd, dtype=dtype)[:, 3 * odd:]
    w = _rand(rng, vocab, dim, dtype=dtype, scale=2 * dim ** -0.5)
    t = rng.integers(0, vocab, rows)
    t[3::4] = rng.choice([-1, vocab, -100, 1 << 40], len(t[3::4]))
    return x, w, torch.from_numpy(t.astype(np.int64)).cuda(), torch.from_numpy(rng.uniform(0.5, 1.5, rows).astype(np.float32)).cuda()


SIZES = [(1, 64, 1), (1, 8, 300), (4, 64, 129), (7, 1, 50), (5, 100, 5000), (64, 128, 256), (65, 64, 255), (130, 200, 700),
         (300, 70, 1025), (1000, 256, 3001), (2100, 128, 6000), (40, 33, 70000), (12300, 1000, 70),
         (70, 1000, 12300)]


@pytest.mark.parametrize("rows,dim,vocab", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [False, True])
def test_loss_and_gradients(rows, dim, vocab, dtype, odd):
    rng = np.random.default_rng(rows + dim + vocab)
    x, w, t, dl = _case(rng, rows, dim, vocab, dtype, odd)
    op = _loss(w, rows)
    losses = op.forward(x, t)
    _check("losses", losses, orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy()), 1e-5)
    out = (t < 0) | (t >= vocab)
    assert (losses[out] == 0).all()
    dx, dw = op.backward(dl)
    wx, ww = orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy(), _np(dl))
    assert (dx[out] == 0).all()
    if vocab == 1:
        assert not dx.any() and not dw.any()
        return
    _check("dx", dx, wx, TOL[dtype])
    _check("dw", dw, ww, TOL[dtype])


def test_no_rows():
    w = torch.randn(300, 64, device="cuda")
    op = _loss(w, 0)
    assert op.forward(torch.empty(0, 64, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0,)
    dx, dw = op.backward(torch.empty(0, device="cuda"))
    assert dx.shape == (0, 64) and not dw.any()


def test_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, w, t, dl = _case(rng, 6, 10, 40, "f32")
    op = _loss(w, 6)
    op.forward(x, t)
    dx, dw = (_np(g) for g in op.backward(dl))
    nx, nw, nt = _np(x), _np(w), t.cpu().numpy()
    f = lambda x, w: float((orc.vocabulary_loss(x, w, nt) * _np(dl)).sum())  # noqa: E731
    for i, j in ((0, 0), (2, 9), (3, 4), (5, 1)):
        d = np.zeros_like(nx)
        d[i, j] = 1e-6
        assert abs((f(nx + d, nw) - f(nx - d, nw)) / 2e-6 - dx[i, j]) < 1e-4
    for i, j in ((0, 0), (int(nt[0]), 3), (39, 9)):
        d = np.zeros_like(nw)
        d[i, j] = 1e-6
        assert abs((f(nx, nw + d) - f(nx, nw - d)) / 2e-6 - dw[i, j]) < 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nearly_certain_targets(dtype):
    """Logits of the target 30 above the others: losses near 1e-11 and their gradients keep their relative size."""
    rng = np.random.default_rng(5)
    rows, dim, vocab = 90, 64, 500
    w = _rand(rng, vocab, dim, dtype=dtype, scale=0.1)
    t = rng.integers(0, vocab, rows)
    target = _np(w)[t]
    # exactly representable x: a multiple of the target's weights would round
    x = torch.from_numpy(np.round(30.0 / (target ** 2).sum(1, keepdims=True) * target * 4) / 4).to(DT[dtype]).cuda()
    t = torch.from_numpy(t).cuda()
    op = _loss(w, rows)
    want = orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy())
    got = _np(op.forward(x, t))
    assert want.max() < 1e-3
    # a logit of about 30 is off by at most 64 roundings of 2^-24 of it: 1.2e-4 of a loss
    assert np.all(np.abs(got - want) <= 1.5e-4 * want + 1e-37)
    dl = torch.ones(rows, device="cuda")
    dx, dw = op.backward(dl)
    wx, ww = orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy(), np.ones(rows))
    _check("dx", dx, wx, TOL[dtype] + 1.5e-4)
    _check("dw", dw, ww, TOL[dtype] + 1.5e-4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_left_out_may_hold_anything(dtype, bad):
    rng = np.random.default_rng(6)
    x, w, t, dl = _case(rng, 70, 64, 400, dtype)
    out = (t < 0) | (t >= 400)
    op = _loss(w, 70)
    want = [op.forward(x, t).clone()] + [g.clone() for g in op.backward(dl)]
    x2, dl2 = x.clone(), dl.clone()
    x2[out] = bad
    dl2[out] = bad
    got = [op.forward(x2, t)] + list(op.backward(dl2))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a bad value in a row that counts stays in its row of dx
    x2 = x.clone()
    x2[0, 5] = bad
    losses = op.forward(x2, t)
    dx, _ = op.backward(dl)
    assert not torch.isfinite(losses[0]) and torch.equal(losses[1:], want[0][1:])
    assert torch.equal(dx[1:], want[1][1:]) and not torch.isfinite(dx[0]).any()


def test_large_logits():
    """Logits of hundreds, of either sign: nothing overflows."""
    rng = np.random.default_rng(7)
    x, w, t, dl = _case(rng, 50, 64, 300, "f32")
    x, w = x * 40, w * 3
    op = _loss(w, 50)
    _check("losses", op.forward(x, t), orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy()), 1e-5)
    dx, dw = op.backward(dl)
    # q's exponent is off by up to 2^-24 of a logit of 1000: 6e-5
    wx, ww = orc.vocabulary_loss(_np(x), _np(w), t.cpu().numpy(), _np(dl))
    _check("dx", dx, wx, 2e-4)
    _check("dw", dw, ww, 2e-4)


@pytest.mark.parametrize("rows,dim,vocab,dtype", [(300, 128, 2000, "bf16"), (5, 64, 30000, "bf16"), (90, 60, 500, "f32")])
def test_replays_of_a_captured_step(rows, dim, vocab, dtype):
    rng = np.random.default_rng(8)
    x, w, t, dl = _case(rng, rows, dim, vocab, dtype)
    op = _loss(w, rows)
    run = lambda: (op.forward(x, t),) + op.backward(dl)  # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for k in range(4):
        x.copy_(_rand(rng, rows, dim, dtype=dtype))
        w.copy_(_rand(rng, vocab, dim, dtype=dtype, scale=2 * dim ** -0.5))
        want = [o.clone() for o in run()]
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        if k % 2:
            torch.cuda.synchronize()
        assert all(torch.equal(o, v) for o, v in zip(outs, want))


def test_another_stream():
    rng = np.random.default_rng(9)
    x, w, t, dl = _case(rng, 200, 96, 900, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = _loss(w, 200), _loss(w, 200)
    got = (a.forward(x, t, stream=side),) + a.backward(dl, stream=side)
    side.synchronize()
    want = (b.forward(x, t),) + b.backward(dl)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
