"""The gated recurrence, the group norm and the loss over a vocabulary at the edges of
their range: workspaces that held NaN, tensors of more than 2^31 elements, tens of
thousands of sequences, a long one among them.

Tolerances: bf16 outputs are fp32 numbers rounded once, 2^-8; fp32 1e-5."""
import os

import numpy as np
import pytest

from conftest import rel_err, rel_max
from oracle import layers as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = 2.0 ** -8 + 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _seq():
    from paper_1902_11208_amd import sequence

    return sequence


def _rand(rng, *shape, dtype=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype).cuda()


def _near(name, a, b, tol):
    a, b = (t.detach().float() for t in (a, b))
    assert a.shape == b.shape, name
    d = (a - b).norm() / b.norm()
    m = (a - b).abs().max() / b.abs().max()
    assert d <= tol and m <= tol, (name, float(d), float(m))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [[30, 0, 100], [9000, 40, 1]], ids=str)
def test_results_unchanged_by_poisoned_workspaces(dtype, lengths):
    rng = np.random.default_rng(1)
    T, C, V = sum(lengths), 40, 300
    z, x, dh = (_rand(rng, T, C, dtype=dtype) for _ in range(3))
    w, t = _rand(rng, V, C, dtype=dtype), torch.from_numpy(rng.integers(-1, V, T)).cuda()
    g, b, dl = _rand(rng, C), _rand(rng, C), torch.rand(T, device="cuda")

    def run():
        s = _seq()
        rec, norm = s.GatedRecurrence(lengths, C, dtype=dtype), s.GroupNorm(lengths, g, b, 5, dtype=dtype, activation="silu")
        loss = s.VocabularyLoss(w, T)
        out = [*rec.forward(z, x, final_state=True), *rec.backward(dh), norm.forward(x), *norm.backward(dh), loss.forward(x, t),
               *loss.backward(dl)]
        return [o.clone() for o in out]

    want = run()
    os.environ["MDLSTM_POISON_WORKSPACE"] = "1"
    try:
        got = run()
    finally:
        del os.environ["MDLSTM_POISON_WORKSPACE"]
    for i, (a, c) in enumerate(zip(got, want)):
        assert torch.equal(a, c) and torch.isfinite(a.float()).all(), i


def test_tensors_beyond_32_bits():
    """40000 tokens of 65536 channels, 2.6 billion elements; the last channels again as a tensor of their own."""
    T, C, lengths = 40000, 65536, [25000, 15000]
    gen = torch.Generator(device="cuda").manual_seed(1)
    z, x, dh = (torch.randn(T, C, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    s = _seq()
    big, small = s.GatedRecurrence(lengths, C), s.GatedRecurrence(lengths, 64)
    last = [v[:, -64:].contiguous() for v in (z, x, dh)]
    h = big.forward(z, x)
    _near("h", h[:, -64:], small.forward(*last[:2]), HALF)
    for name, a, b in zip(("dz", "dx"), big.backward(dh), small.backward(last[2])):
        _near(name, a[:, -64:], b, HALF)
    del big, h
    torch.cuda.empty_cache()
    w, b = torch.randn(C, generator=gen, device="cuda"), torch.randn(C, generator=gen, device="cuda")
    big, small = s.GroupNorm(lengths, w, b, 1024, activation="silu"), s.GroupNorm(lengths, w[-64:].clone(), b[-64:].clone(), 1, activation="silu")
    _near("y", big.forward(x)[:, -64:], small.forward(last[1]), HALF)
    got, want = big.backward(dh), small.backward(last[2])
    _near("dx", got[0][:, -64:], want[0], HALF)
    for a, c in zip(got[1:], want[1:]):
        _near("dw, db", a[-64:], c, 1e-4)


def test_weights_beyond_32_bits():
    """1.1 million tokens of 2048 numbers; losses and gradients against products of pieces of the vocabulary in fp32."""
    rows, dim, vocab = 66, 2048, 1_100_000
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, dim, generator=gen, device="cuda").bfloat16()
    w = torch.randn(vocab, dim, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(2.0 / dim ** 0.5)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t[0], t[1], t[2] = vocab - 1, 0, vocab
    dl = torch.rand(rows, generator=gen, device="cuda") + 0.5
    op = _seq().VocabularyLoss(w, rows)
    losses = op.forward(x, t)
    dx, dw = op.backward(dl)
    logits = torch.cat([x.float() @ c.float().t() for c in w.split(100_000)], 1).double()
    ok, at = t < vocab, t.clamp(max=vocab - 1)
    lse = torch.logsumexp(logits, 1)
    want = torch.where(ok, lse - logits.gather(1, at[:, None])[:, 0], 0.0)
    assert float((losses - want).abs().max()) < 1e-5 * float(want.abs().max())
    q = torch.exp(logits - lse[:, None])
    q.scatter_add_(1, at[:, None], torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda"))
    q = (q * (dl * ok)[:, None]).float()
    _near("dx", dx, sum(a @ c.float() for a, c in zip(q.split(100_000, 1), w.split(100_000))), 2 * HALF)
    for rows_of in (t[:2], torch.arange(vocab - 300, vocab, device="cuda"), t[3:]):
        _near("dw", dw[rows_of], q[:, rows_of].t() @ x.float(), 2 * HALF)


@pytest.mark.parametrize("lengths", [np.ones(70000, np.int64), np.r_[np.tile([0, 3, 1], 1700), 9000, np.tile([2, 5], 900)]],
                         ids=["70000 of one token", "a long one among thousands"])
def test_many_sequences(lengths):
    rng = np.random.default_rng(3)
    T, C = int(lengths.sum()), 8
    z, x, dh = (_rand(rng, T, C) for _ in range(3))
    nz, nx, nd = (t.cpu().numpy().astype(np.float64) for t in (z, x, dh))
    op = _seq().GatedRecurrence(lengths, C, dtype=torch.float32)
    h, final = op.forward(z, x, final_state=True)
    wh, wf = orc.recurrence_forward(nz, nx, lengths, "sigmoid")
    for name, a, b in (("h", h, wh), ("final", final, wf), *zip(("dz", "dx"), op.backward(dh), orc.recurrence_backward(nz, nx, lengths, "sigmoid", nd))):
        assert rel_err(a.cpu().numpy(), b) < 1e-5 and rel_max(a.cpu().numpy(), b) < 1e-5, name
    w, b = _rand(rng, C), _rand(rng, C)
    norm = _seq().GroupNorm(lengths, w, b, 2, dtype=torch.float32)
    y = norm.forward(x)
    args = (lengths, w.cpu().numpy(), b.cpu().numpy(), 2, 1e-5, None)
    assert rel_err(y.cpu().numpy(), orc.group_norm(nx, *args)) < 1e-5
    # groups of four values: dx is a difference of numbers of |g| / dev, dev down to sqrt(eps): 2^-24 of them, some ten roundings
    dx, dw, db = (t.cpu().numpy() for t in norm.backward(dh))
    wx, ww, wb = orc.group_norm(nx, *args, dy=nd)
    assert np.abs(dx - wx).max() <= 1e-6 * np.abs(nd).max() * np.abs(args[1]).max() / np.sqrt(1e-5)
    assert rel_err(dw, ww) < 1e-4 and rel_err(db, wb) < 1e-4
