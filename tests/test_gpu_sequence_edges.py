"""GPU checks of the sequence operators at the edges of their range, against the
float64 oracle (oracle/sequence.py): values that are not finite in long
sequences, an object's own outputs as its inputs, sizes beyond 2^32 threads,
streams.

Tolerances, normwise L2 and max-norm relative error: 1e-5 for fp32 storage; for
bf16 storage 3 * 2^-8 (an output is rounded once and computed from at most two
operands rounded to bf16), and 2^-7 for fp32 results of bf16 inputs."""
import numpy as np
import pytest

from conftest import rel_err, rel_max
from oracle import sequence as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = {"f32": 1e-5, "bf16": 3 * 2.0 ** -8}
TOL32 = {"f32": 1e-5, "bf16": 2.0 ** -7}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _seq():
    from paper_1902_11208_amd import sequence

    return sequence


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _check(name, got, want, tol):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    e, m = rel_err(got, want), rel_max(got, want)
    assert e <= tol and m <= tol, (name, e, m)


def _rand(rng, *shape, dtype="f32"):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype,d", [("f32", 16), ("f32", 64), ("bf16", 32), ("bf16", 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_gradients_before_a_bad_value_in_a_later_segment(dtype, d, bad):
    """2500 tokens are cut into segments of 128. From the end, token 276 is the 21st of a segment: the 20 that the
    scan meets before it in that segment see nothing of its bad value, but share a chunk's products with it."""
    rng = np.random.default_rng(d)
    T, heads, at = 2500, 2, 276
    print(f"case: bad value in a segment, {dtype}, {d} columns, {bad}", flush=True)
    q, k, v, do = (_rand(rng, T, heads, d, dtype=dtype) for _ in range(4))
    a = torch.tensor([0.1, 0.2], device="cuda")
    op = _seq().DecayAttention([T], heads, d, d, a, dtype=DT[dtype])
    _, wk, wv, _ = orc.attention_backward(_np(q), _np(k), _np(v), [T], _np(a), d ** -0.5, _np(do))
    q2, do2 = q.clone(), do.clone()
    q2[T - 1 - at, 1, 5] = do2[T - 1 - at, 1, 5] = bad
    rows = slice(T - at, T - 256)
    op.forward(q2, k, v)
    dk = op.backward(do)[1].clone()
    _check("dk", dk[rows, 1, 5], wk[rows, 1, 5], TOL[dtype])
    op.forward(q, k, v)
    dv = op.backward(do2)[2].clone()
    _check("dv", dv[rows, 1, 5], wv[rows, 1, 5], TOL[dtype])
    for got, want in ((dk, wk), (dv, wv)):
        assert torch.isfinite(got[T - at:]).all() and not torch.isfinite(got[:T - at, 1, 5]).any()
        _check("other columns", got[:, :, :5], want[:, :, :5], TOL[dtype])
