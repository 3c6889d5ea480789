"""The gated recurrence with coefficients given (gate None), where products of factors leave fp32's range and the
recurrence does not, or the other way round: what it gives token by token, in 64 bits from the same fp32 factors.

Tolerances. A state is a product of at most T factors (u is 0 but where a state starts), each product rounded at 2^-24 of
itself, and joined from products of slices rounded as often: 2 T 2^-24 of itself. Factors are chosen so that no state
lies below fp32's normal range, where a rounding would be larger."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _walk(f, u, h):
    """h of every token, from fp32 coefficients [T, C] in 64 bits; beyond fp32's largest number infinite, as there."""
    out, h = np.empty(f.shape), h.astype(np.float64)
    with np.errstate(all="ignore"):
        for t in range(len(f)):
            h = f[t].astype(np.float64) * h + u[t]
            h = np.where(np.abs(h) > np.finfo(np.float32).max, np.sign(h) * np.inf, h)
            out[t] = h
    return out


def _check(name, got, want, T):
    got = got.cpu().numpy().astype(np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(all="ignore"):
        near = np.abs(got - want) <= 2 * T * 2.0 ** -24 * np.abs(want)
    bad = np.argwhere(~(same | near))
    assert len(bad) == 0, (name, len(bad), bad[0], got[tuple(bad[0])], want[tuple(bad[0])])


def _both_ways(f, u, state):
    """h, the final state and the adjoint (the same recurrence from the end: s_t = f_t (dh_t + s_(t+1)))."""
    from paper_1902_11208_amd import sequence

    T, C = f.shape
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    op = sequence.GatedRecurrence([T], C, dtype=torch.float32, gate=None)
    h, final = op.forward(cuda(f), cuda(u), state=cuda(state[None]), final_state=True)
    want = _walk(f, u, state)
    _check("h", h, want, T)
    _check("final", final[0], want[-1], T)
    zero = np.zeros_like(f)
    op.forward(cuda(f[::-1]), cuda(zero), state=cuda(zero[:1]))
    # dx_t = dh_t + s_(t+1) and s_t = f_t dx_t, so with dh = 0 the adjoint before token t is f_t dx_t
    _, dx, dstate = op.backward(cuda(zero), cuda(state[None]))
    want = _walk(f, zero, state)
    _check("dstate", dstate[0], want[-1], T)
    _check("dx", dx.flip(0)[1:], want[:-1], T)


@pytest.mark.parametrize("at", [0, 3, 8, 120, 130, 500])
@pytest.mark.parametrize("T", [600, 5000])
def test_out_of_the_range_and_back_within_a_slice(T, at):
    """Eight factors whose product is 1, and whose partial products are far below fp32's range, or beyond it."""
    f = np.ones((T, 6), np.float32)
    state = np.array([1e12, 1e12, 1e3, 1e3, 1e12, 1.0], np.float32)
    for c, (lo, hi) in enumerate([(1e-12, 1e12), (1e-12, 1e12), (1e10, 1e-10), (1e10, 1e-10), (1e-6, 1e6), (1e9, 1e-9)]):
        gap = (0, 0, 0, 5, 3, 0)[c]
        f[at:at + 4, c], f[at + 4 + gap:at + 8 + gap, c] = lo, hi
    f[:, 1] = f[:, 0][::-1]
    _both_ways(f, np.zeros_like(f), state)


@pytest.mark.parametrize("T", [1000, 1700, 20000])
def test_slow_falls_and_rises(T):
    """States that go down to 2^-115 and up to 2^36 in waves of 5 tokens to several tiles and segments."""
    C = 24
    t = np.arange(-1, T)[:, None]
    rng = np.random.default_rng(T)
    period = np.exp(rng.uniform(np.log(5), np.log(6000), C))
    y = -39.5 + 75.5 * np.cos(2 * np.pi * t / period)
    f = np.exp2(y[1:] - y[:-1]).astype(np.float32)
    f *= np.where(rng.random(f.shape) < 0.3, -1, 1).astype(np.float32)
    state = np.exp2(y[0]).astype(np.float32)
    _both_ways(f, np.zeros_like(f), state)


@pytest.mark.parametrize("T,first", [(1000, 0), (1000, 300), (6000, 0), (6000, 2000)])
def test_a_fall_of_a_few_tokens_and_a_long_rise(T, first):
    """A state, or an input where there was none, falls by 2^158 in twelve or twenty tokens; factors of 1.18, slices of
    which grow by less than 4, bring it back hundreds of tokens and several segments later."""
    C = 4
    f, u, state = np.ones((T, C), np.float32), np.zeros((T, C), np.float32), np.zeros(C, np.float32)
    for c, n in enumerate((12, 20, 12, 20)):
        f[first + 1:first + 1 + n, c] = np.float32(2.0 ** (-158 / n))
        f[first + 1 + n:first + 600, c] = 1.18
        if c < 2:
            state[c] = 2.0 ** 39
        else:
            u[first, c] = 2.0 ** 39
    _both_ways(f, u, state)
