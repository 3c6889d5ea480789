"""The group norm's relu lets through backward what it let through forward, also where u is 0 but for its rounding."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("lengths", [[60], [40, 0, 200], [9000, 5]], ids=str)
@pytest.mark.parametrize("channels,groups", [(512, 32), (320, 5), (66, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_mask_is_the_forward_pass_own(lengths, channels, groups, dtype):
    """With dy of ones, db counts what came through (whole numbers below 2^24, exact in fp32): as many as outputs above 0.
    A third of the tokens hold one row, and the bias takes its u to 0 but for the rounding."""
    from paper_1902_11208_amd import sequence

    rng = np.random.default_rng(channels)
    T = sum(lengths)
    x = torch.from_numpy(rng.standard_normal((T, channels)).astype(np.float32)).to(dtype).cuda()
    x[::3] = x[0]
    w = torch.from_numpy(rng.uniform(0.5, 2.0, channels).astype(np.float32)).cuda()
    # u of that row in 64 bits from the first sequence's statistics, rounded: what the kernels come near in fp32
    first = x[:lengths[0]].double().view(lengths[0], groups, -1)
    mean, var = first.mean((0, 2), keepdim=True), first.var((0, 2), unbiased=False, keepdim=True)
    b = -(((first[:1] - mean) / (var + 1e-5).sqrt()).view(-1) * w.double()).float()
    op = sequence.GroupNorm(lengths, w, b, groups, dtype=dtype, activation="relu")
    y = op.forward(x).clone()
    _, _, db = op.backward(torch.ones_like(x))
    assert torch.equal(db, (y > 0).sum(0).float())
