"""Every number of the group norm and its gradients against the float64 oracle (oracle/layers.py), within what the
roundings of the computation in fp32 come to, R = 2^-24 each: also where gradients cancel (groups of a few values, weights
whose sums are near 0).

A sum over a group goes through at most K = 170 additions one after another: 32 tokens of a thread, 64 slices of a
workgroup, 70 for a group's channels (4096 of them by a wave); segments are joined in 64 bits. So it is K R of the sum of
magnitudes off. From there on each bound below follows the formula that it stands by: d = x - mean, c = d rstd,
u = c w + b, e = dy act'(u), g = e w, dx = rstd (g - mean(g) - c mean(g c)). bf16 outputs are rounded once more, 2^-8."""
import numpy as np
import pytest

from oracle import layers as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

R, K, EPS = 2.0 ** -24, 170, 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(built_lib):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _bounds(x, dy, lengths, w, b, groups, act):
    """The bounds of y, dx, dw and db."""
    C = x.shape[1]
    oy, ox, ow, ob = np.zeros_like(x), np.zeros_like(x), np.zeros(C), np.zeros(C)
    t = 0
    for n in lengths:
        at = slice(t, t + int(n))
        t += int(n)
        if n == 0:
            continue
        of = lambda v: v.reshape(-1, groups, C // groups)  # noqa: E731
        mean_of = lambda v: of(v).mean((0, 2), keepdims=True)  # noqa: E731
        spread = lambda v: np.broadcast_to(v, of(x[at]).shape).reshape(-1, C)  # noqa: E731
        v, mean = x[at], mean_of(x[at])
        d = v - spread(mean)
        rstd = spread(1 / np.sqrt(mean_of(d * d) + EPS))
        c = d * rstd
        u = c * w + b
        off_mean = spread(2 * R * np.abs(mean) + (K + 2) * R * mean_of(np.abs(d)))  # found once, then corrected by the distances' mean
        off_r = (K / 2 + 6) * R  # relative: half of the variance's, the root's and the quotient's
        off_c = rstd * (off_mean + R * np.abs(d)) + (off_r + R) * np.abs(c)
        off_u = np.abs(w) * off_c + 2 * R * (np.abs(c * w) + np.abs(b))
        s = 1 / (1 + np.exp(-u))
        if act == "silu":  # |act'| <= 1.1, |act''| <= 1/2; the sigmoid and its products within 16 roundings
            oy[at] = 1.1 * off_u + 16 * R * np.abs(u * s)
            slope, off_slope = s * (1 + u * (1 - s)), off_u / 2 + 16 * R * s * (1 + np.abs(u))
        else:
            oy[at], slope, off_slope = off_u + R * np.abs(u), np.ones_like(u), np.zeros_like(u)
        e, off_e = dy[at] * slope, np.abs(dy[at]) * (off_slope + R * np.abs(slope))
        g, off_g = e * w, np.abs(w) * off_e + R * np.abs(e * w)
        mg, off_mg = spread(mean_of(g)), spread(mean_of(off_g) + (K + 2) * R * mean_of(np.abs(g)))
        mgc = spread(mean_of(g * c))
        off_gc = np.abs(g) * off_c + np.abs(c) * off_g
        off_mgc = spread(mean_of(off_gc) + (K + 3) * R * mean_of(np.abs(g * c)))
        size = np.abs(g) + np.abs(mg) + np.abs(c * mgc)
        ox[at] = rstd * (off_g + off_mg + np.abs(c) * off_mgc + off_c * np.abs(mgc) + (4 * R + off_r) * size)
        # sums over all tokens: 4096 workgroups' shares more, 64 slices of 64 and more of them
        ow += (off_e * np.abs(c) + np.abs(e) * off_c + (K + 160) * R * np.abs(e * c)).sum(0)
        ob += (off_e + (K + 160) * R * np.abs(e)).sum(0)
    return oy, ox, ow, ob


@pytest.mark.parametrize("lengths", [[1], [2, 0, 3, 1], [127, 128, 1, 0, 9], [700, 30], [5000, 2, 0, 3000], [1] * 5000 + [4000]],
                         ids=lambda v: str(v) if len(v) < 9 else "thousands and a long one")
@pytest.mark.parametrize("channels,groups", [(1, 1), (6, 2), (40, 40), (320, 32), (300, 1), (520, 130)])
@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_number(lengths, channels, groups, act, dtype):
    from paper_1902_11208_amd import sequence

    rng = np.random.default_rng(channels + len(lengths))
    T = sum(lengths)
    new = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    x, dy = (new(T, channels) + 0.5).to(dtype).cuda(), new(T, channels).to(dtype).cuda()
    w, b = (1 + 0.3 * new(channels)).cuda(), (0.3 * new(channels)).cuda()
    op = sequence.GroupNorm(lengths, w, b, groups, dtype=dtype, eps=EPS, activation=act)
    got = [op.forward(x).clone(), *op.backward(dy)]
    nx, ndy, nw, nb = (v.cpu().to(torch.float64).numpy() for v in (x, dy, w, b))
    eps = float(np.float32(EPS))
    want = [orc.group_norm(nx, lengths, nw, nb, groups, eps, act), *orc.group_norm(nx, lengths, nw, nb, groups, eps, act, dy=ndy)]
    for name, a, ref, off in zip(("y", "dx", "dw", "db"), got, want, _bounds(nx, ndy, lengths, nw, nb, groups, act)):
        if dtype == torch.bfloat16 and name in ("y", "dx"):
            off = off + 2.0 ** -8 * (np.abs(ref) + off)
        bad = np.abs(a.cpu().to(torch.float64).numpy() - ref) / (off + 1e-300)
        bad = np.where((off == 0) & (bad == 0), 0, bad)
        assert bad.max(initial=0) <= 1, (name, bad.max(), np.unravel_index(bad.argmax(), bad.shape))
