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


@pytest.mark.parametrize("lengths,d,dtype", [([33, 0, 70], 32, "f32"), ([33, 0, 70], 64, "bf16"), ([1500, 900], 64, "f32"),
                                             ([1500, 900], 128, "bf16")])
def test_states_of_an_object_passed_back_to_it(lengths, d, dtype):
    """Three pieces of the same sequences through one object, whole and in segments: each piece starts from the states
    that the one before left, each backward call takes the state gradients that the one before gave."""
    rng = np.random.default_rng(sum(lengths) + d)
    T, n, heads = sum(lengths), len(lengths), 2
    print(f"case: three pieces of {lengths}, {d} columns, {dtype}", flush=True)
    a = torch.from_numpy(rng.uniform(0.01, 0.1, heads).astype(np.float32)).cuda()
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    state, dstate = _rand(rng, n, heads, d, d), _rand(rng, n, heads, d, d)
    for piece in range(3):
        q, k, v, do = (_rand(rng, T, heads, d, dtype=dtype) for _ in range(4))
        before = state.clone()
        args = _np(q), _np(k), _np(v), lengths, _np(a), d ** -0.5
        o, final = op.forward(q, k, v, state=state, final_state=True)
        wo, wf = orc.attention_forward(*args, _np(before))
        _check("o", o, wo, TOL[dtype])
        _check("final", final, wf, TOL32[dtype])
        assert torch.equal(state, before), "the call wrote to its own input"
        for _ in range(2):
            given = dstate.clone()
            *grads, ds = op.backward(do, dstate=dstate)
            want = orc.attention_backward(*args, _np(do), _np(before), _np(given))
            for name, g, w in zip(("dq", "dk", "dv"), grads, want):
                _check(name, g, w, TOL[dtype])
            _check("dstate", ds, want[3], TOL32[dtype])
            assert torch.equal(dstate, given), "the call wrote to its own input"
            dstate = ds
        state = final


def test_attention_refuses_its_other_outputs_as_inputs():
    """Outputs and gradients of an object as its own inputs, which workgroups would read and write in no order."""
    from paper_1902_11208_amd import MdlstmError

    op = _seq().DecayAttention([40, 30], 2, 32, 32, torch.zeros(2, device="cuda"), dtype=torch.float32)
    q = torch.ones(70, 2, 32, device="cuda")
    o = op.forward(q, q, q)
    for args in ((o, q, q), (q, o, q), (q, q, o)):
        with pytest.raises(MdlstmError, match="o overlaps"):
            op.forward(*args)
    dq, dk, dv = op.backward(o)  # o is no output of that call
    for g in (dq, dk, dv):
        with pytest.raises(MdlstmError, match="overlaps grad_o"):
            op.backward(g)


def _same_kind(name, got, want, tol):
    """NaN and infinities where `want` has them, the rest within the tolerance."""
    got = _np(got)
    for what in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(what(got), what(want)), (name, what.__name__, int(what(got).sum()), int(what(want).sum()))
    f = np.isfinite(want)
    _check(name, np.where(f, got, 0), np.where(f, want, 0), tol)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("where", ["q", "k", "v", "do", "state", "dstate"])
@pytest.mark.parametrize("lengths,d,dtype", [([90, 45], 16, "f32"), ([90, 45], 32, "f32"), ([90, 45], 64, "bf16"),
                                             ([90, 45], 128, "bf16"), ([1000], 64, "f32"), ([1000], 64, "bf16")])
def test_infinite_values_give_what_the_recurrence_gives(lengths, d, dtype, where, bad):
    """One value that is not finite, early in the first sequence: outputs, states and gradients are infinite or NaN
    where the recurrence in 64 bits is, whole and in segments of 128."""
    rng = np.random.default_rng(d + len(lengths))
    T, n, heads = sum(lengths), len(lengths), 2
    print(f"case: {bad} in {where}, {lengths}, {d} columns, {dtype}", flush=True)
    t = {x: _rand(rng, T, heads, d, dtype=dtype) for x in ("q", "k", "v", "do")}
    t["state"], t["dstate"] = _rand(rng, n, heads, d, d), _rand(rng, n, heads, d, d)
    t[where][(0, 1, 3, 5) if "state" in where else (20, 1, 5)] = bad
    a = torch.tensor([0.02, 0.05], device="cuda")
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    o, final = op.forward(t["q"], t["k"], t["v"], state=t["state"], final_state=True)
    got = op.backward(t["do"], dstate=t["dstate"])
    args = _np(t["q"]), _np(t["k"]), _np(t["v"]), lengths, _np(a), d ** -0.5
    with np.errstate(invalid="ignore"):
        wo, wf = orc.attention_forward(*args, _np(t["state"]))
        want = orc.attention_backward(*args, _np(t["do"]), _np(t["state"]), _np(t["dstate"]))
    _same_kind("o", o, wo, TOL[dtype])
    _same_kind("final", final, wf, TOL32[dtype])
    for name, g, w in zip(("dq", "dk", "dv", "dstate"), got, want):
        _same_kind(name, g, w, TOL32[dtype] if name == "dstate" else TOL[dtype])


@pytest.mark.parametrize("lengths,d,dtype", [([200, 33], 32, "f32"), ([200, 33], 64, "bf16"), ([1000], 64, "bf16"),
                                             ([1000], 128, "f32")])
def test_states_near_the_largest_number(lengths, d, dtype):
    """States of some 2^124, of which fp32 holds 2^128, with outputs of ordinary size."""
    rng = np.random.default_rng(d)
    T, n, heads = sum(lengths), len(lengths), 2
    q, k, v = (_rand(rng, T, heads, d, dtype=dtype) * s for s in (2.0 ** -120, 2.0 ** 61, 2.0 ** 61))
    a, st = torch.tensor([0.05, 0.1], device="cuda"), _rand(rng, n, heads, d, d) * 2.0 ** 122
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    o, final = op.forward(q, k, v, state=st, final_state=True)
    wo, wf = orc.attention_forward(_np(q), _np(k), _np(v), lengths, _np(a), d ** -0.5, _np(st))
    assert np.abs(wf).max() < 2.0 ** 127
    _check("o", o, wo, TOL[dtype])
    _check("final", final, wf, TOL32[dtype])


# --- more than 2^32 threads along one dimension of a grid, which the runtime does not take ---------------------
def _room(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GiB of device memory")


def _randn(*shape, seed=1):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


def test_dropout_of_more_rows_than_threads():
    """2^32 + 3 rows of one element, a thread each: rows two apart, so they are not one long row."""
    _room(40)
    rows, p, seed, call = (1 << 32) + 3, 0.5, 7, 9
    x = torch.ones(rows, 2, dtype=torch.bfloat16, device="cuda")[:, :1]
    y = _seq().dropout(x, p, seed, call)[:, 0]
    kept = int((y[:1 << 31] == 2).sum()), int((y[1 << 31:] == 2).sum())
    assert all(abs(k - (1 << 30)) < 5 * 2 ** 15.5 for k in kept), kept
    for e in (0, 1 << 31, 1 << 32):  # element e = 8 b + j has half j of block b's words
        w = [h for x in orc.philox(e >> 3, call, seed) for h in (x & 0xFFFF, x >> 16)]
        assert [float(v) for v in y[e:e + 3]] == [2.0 if u >= 1 << 15 else 0.0 for u in w[:3]], e
    del x, y
    torch.cuda.empty_cache()


def test_norm_of_more_rows_than_workgroups():
    """2^29 + 1 rows of one element, eight threads each."""
    _room(16)
    rows = (1 << 29) + 1
    x = _randn(rows, 1)
    y, _ = _seq().ResidualNorm(torch.ones(1, device="cuda"), rows, eps=1.0).forward(x)
    for at in range(0, rows, 1 << 27):
        a = x[at:at + (1 << 27)].float()
        assert float((y[at:at + (1 << 27)].float() - a * torch.rsqrt(a * a + 1)).abs().max()) <= 2.0 ** -8
    del x, y
    torch.cuda.empty_cache()


def test_attention_of_more_examples_than_workgroups():
    """16400 examples of one token with 1024 heads, a workgroup of 256 threads each."""
    _room(16)
    n, heads, d = 16400, 1024, 33
    q, k, v = (_randn(n, heads, d, seed=s) for s in (1, 2, 3))
    op = _seq().DecayAttention(np.ones(n, np.int64), heads, d, d, torch.zeros(heads, device="cuda"), scale=1.0)
    o = op.forward(q, k, v)
    for at in range(0, n, 4100):
        s = slice(at, at + 4100)
        want = (q[s].float() * k[s].float()).sum(2, keepdim=True) * v[s].float()
        assert float((o[s].float() - want).norm() / want.norm()) <= TOL["bf16"]
    del q, k, v, o, op
    torch.cuda.empty_cache()


def test_states_of_more_examples_than_workgroups():
    """One example of 1500 tokens in segments among 65600 empty ones of 256 heads, which keep their states; steps of
    2^24 rows, the most of one call."""
    _room(16)
    rng = np.random.default_rng(31)
    n, heads, d, T = 65601, 256, 4, 1500
    lengths = np.zeros(n, np.int64)
    lengths[n - 1] = T
    q, k, v = (_rand(rng, T, heads, d) for _ in range(3))
    a = torch.from_numpy(rng.uniform(0, 0.1, heads).astype(np.float32)).cuda()
    st = torch.randn(n, heads, d, d, device="cuda")
    o, final = _seq().DecayAttention(lengths, heads, d, d, a, dtype=torch.float32).forward(q, k, v, state=st, final_state=True)
    wo, wf = orc.attention_forward(_np(q), _np(k), _np(v), [T], _np(a), d ** -0.5, _np(st[-1:]))
    _check("o", o, wo, 1e-5)
    _check("final", final[-1:], wf, 1e-5)
    assert torch.equal(final[:-1], st[:-1])
    n = 1 << 24
    q, k, v, st = (torch.randn(n, 1, 1, device="cuda") for _ in range(4))
    st = st.unsqueeze(3)
    want = st * 0.5 + (k * v).unsqueeze(3)
    o = _seq().decay_attention_step(q, k, v, st, torch.tensor([np.log(2.0)], dtype=torch.float32, device="cuda"), scale=1.0)
    assert float((st - want).abs().max()) <= 1e-5 and float((o - q * want[:, :, 0]).abs().max()) <= 1e-4


def test_gradients_of_shared_heads_beyond_32_bits():
    """2^32 elements of dk, each summed over the two heads that share it. A rate of 200 leaves nothing of the token
    before, so dk = scale (q_0 (do_0 . v) + q_1 (do_1 . v)) of the token itself."""
    _room(120)
    T, kv, dk = 65544, 512, 128
    q, do, k, v = _randn(T, 2 * kv, dk), _randn(T, 2 * kv, 1, seed=2), _randn(T, kv, dk, seed=3), _randn(T, kv, 1, seed=4)
    op = _seq().DecayAttention([4096] * 16 + [8], 2 * kv, dk, 1, torch.full((2 * kv,), 200.0, device="cuda"), kv_heads=kv, scale=1.0)
    op.forward(q, k, v)
    got = op.backward(do)[1]
    for at in (0, 32768, T - 64):
        s = slice(at, at + 64)
        want = (q[s].float() * do[s].float()).unflatten(1, (kv, 2)).sum(2) * v[s].float()
        assert float((got[s].float() - want).norm() / want.norm()) <= TOL["bf16"]
        assert torch.isfinite(got[s]).all()
    del q, do, k, v, op, got
    torch.cuda.empty_cache()


# --- streams -----------------------------------------------------------------------------------------------------
def test_buffers_of_another_stream():
    """Fresh objects called with stream=: memory that the current stream has freed, but still writes, must not become
    their buffers. Blocks of the buffers' sizes are freed while fills of them wait behind a long kernel."""
    rng = np.random.default_rng(37)
    T, heads, d = 300, 2, 64
    sq, side = _seq(), torch.cuda.Stream()
    q, k, v, do = (_rand(rng, T, heads, d) for _ in range(4))
    st, ds, a = _rand(rng, 1, heads, d, d), _rand(rng, 1, heads, d, d), torch.tensor([0.05, 0.1], device="cuda")
    x, res, dy, w = _rand(rng, T, 128), _rand(rng, T, 128), _rand(rng, T, 128), torch.ones(128, device="cuda")

    def calls(stream):
        op = sq.DecayAttention([T], heads, d, d, a, dtype=torch.float32)
        norm = sq.ResidualNorm(w, T, dtype=torch.float32, dropout=0.2)
        norm8 = sq.ResidualNorm(w, T, dtype=torch.float32, out="fp8")
        state = st.clone()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
            torch.cuda._sleep(100_000_000)  # some 50 ms
            for n in (T * heads * d, heads * d * d, T * 128, T, 128, T * 32, T * 128 // 4, 64, 4096, 1 << 16):
                blocks = [torch.empty(n, device="cuda") for _ in range(8)]
                for b in blocks:
                    b.fill_(float("nan"))
                del blocks, b
        y, h = norm.forward(x, res, seed=1, call=2, stream=stream)
        y8, scale, _ = norm8.forward(x, res, stream=stream)
        got = [*op.forward(q, k, v, state=st, final_state=True, stream=stream), *op.backward(do, dstate=ds, stream=stream),
               y, h, *norm.backward(dy, dy, stream=stream), y8.view(torch.uint8), scale,
               sq.dropout(x, 0.5, 3, 4, stream=stream),
               sq.decay_attention_step(q[:1], k[:1], v[:1], state, a, stream=stream)]
        return got, (op, norm, norm8, state)

    want, keep = calls(None)
    torch.cuda.synchronize()
    got, keep2 = calls(side)
    torch.cuda.synchronize()
    for i, (g, w_) in enumerate(zip(got, want)):
        assert torch.equal(g, w_), i


# --- norm ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("cols,dtype", [(64, "f32"), (512, "bf16"), (3000, "bf16")])
def test_norm_of_its_own_output(cols, dtype):
    """A norm's y as its next x, without residual and dropout, where h is x: the gradients need what x was."""
    rng = np.random.default_rng(cols)
    x, dy = _rand(rng, 5, cols, dtype=dtype), _rand(rng, 5, cols, dtype=dtype)
    w = 1 + 0.3 * _rand(rng, cols)
    op = _seq().ResidualNorm(w, 5, dtype=DT[dtype], eps=1e-5)
    y, _ = op.forward(x)
    h = y.clone()
    y, got_h = op.forward(y)
    dx, _, dw = op.backward(dy)
    _check("y", y, orc.norm_forward(_np(h), _np(w), 1e-5)[0], TOL[dtype])
    wx, _, ww = orc.norm_backward(_np(h), _np(w), 1e-5, _np(dy))
    assert torch.equal(got_h, h)
    _check("dx", dx, wx, TOL[dtype])
    _check("dw", dw, ww, TOL32[dtype])


@pytest.mark.parametrize("t", [13, 19, 26, 31, 38, 51, 62, 95, 125, 3001])
def test_fp8_codes_are_those_of_the_quotient(t):
    """h = 1/2 everywhere and eps = 3/4 make the norm's factor 1 and y = w / 2, exactly. Quotients y / scale lie at
    ties of e4m3 or one rounding beside them: the codes are those of the fp32 quotient."""
    num = torch.arange(1, 128, 2, dtype=torch.float32)
    w = torch.cat([torch.full((1,), 128.0), num]) * t * 2.0 ** -8
    x = torch.full((3, w.numel()), 0.5, device="cuda")
    y8, scale, _ = _seq().ResidualNorm(w.cuda(), 3, dtype=torch.float32, eps=0.75, out="fp8").forward(x)
    y = w * 0.5
    s = y[0] / torch.tensor(448.0)
    assert torch.equal(scale.cpu(), s.expand(3))
    want = (y / s).to(torch.float8_e4m3fn)
    got = y8.cpu()
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8).expand(3, -1)), (got.float()[0] - want.float()).nonzero()


# --- bf16 --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("lengths,heads,kv,dk,dv", [([300, 0, 131], 4, 4, 32, 32), ([300, 131], 4, 2, 64, 64),
                                                    ([300, 131], 4, 1, 128, 128), ([200, 77], 2, 2, 24, 100), ([1500], 2, 2, 64, 64)])
def test_bf16_outputs_are_rounded_once(lengths, heads, kv, dk, dv):
    """Scores and states enter the products as fp32 numbers, so outputs and gradients carry the error of their own
    rounding only: uniform in half a step of 8 bits either way, that is 2^-7 / sqrt(12) of the binade's lower edge or
    less, in the mean over many outputs. Shared heads' sums and states see fp32 sums too."""
    rng = np.random.default_rng(dk + dv)
    T, n, once = sum(lengths), len(lengths), 2.0 ** -7 / 12 ** 0.5
    print(f"case: bf16 {lengths} heads {heads}/{kv} dims {dk}x{dv}", flush=True)
    q, k = _rand(rng, T, heads, dk, dtype="bf16"), _rand(rng, T, kv, dk, dtype="bf16")
    v, do = _rand(rng, T, kv, dv, dtype="bf16"), _rand(rng, T, heads, dv, dtype="bf16")
    st, ds = _rand(rng, n, heads, dk, dv), _rand(rng, n, heads, dk, dv)
    a = torch.from_numpy(rng.uniform(0.004, 0.3, heads).astype(np.float32)).cuda()
    op = _seq().DecayAttention(lengths, heads, dk, dv, a, kv_heads=kv)
    o, final = op.forward(q, k, v, state=st, final_state=True)
    dq, dk_, dv_, dst = op.backward(do, dstate=ds)
    args = _np(q), _np(k), _np(v), lengths, _np(a), dk ** -0.5
    wo, wf = orc.attention_forward(*args, _np(st))
    want = orc.attention_backward(*args, _np(do), _np(st), _np(ds))
    for name, g, w in zip(("o", "dq", "dk", "dv"), (o, dq, dk_, dv_), (wo, *want[:3])):
        assert rel_err(_np(g), w) <= once, (name, rel_err(_np(g), w))
    for name, g, w in (("final", final, wf), ("dstate", dst, want[3])):
        assert rel_err(_np(g), w) <= 1e-5, (name, rel_err(_np(g), w))


def test_streams_by_their_handle():
    """stream= takes whatever holds a stream's handle (the default stream's is 0)."""
    import types

    side = torch.cuda.Stream()
    x = torch.ones(40, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    want = _seq().ResidualNorm(w, 40, dtype=torch.float32).forward(x)[0]
    drop = _seq().dropout(x, 0.5, 1)
    torch.cuda.synchronize()
    for s in (torch.cuda.default_stream(), side, types.SimpleNamespace(cuda_stream=side.cuda_stream),
              torch.cuda.ExternalStream(side.cuda_stream)):
        y = _seq().ResidualNorm(w, 40, dtype=torch.float32).forward(x, stream=s)[0]
        d = _seq().dropout(x, 0.5, 1, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(d, drop)
