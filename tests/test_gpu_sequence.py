"""GPU parity of the sequence operators (linear attention with decay, its
single-token step, residual norm with its 8-bit output, dropout) against the
float64 oracle (oracle/sequence.py).

Tolerances per tensor, normwise L2 and max-norm relative error. fp32 storage:
1e-5, as for the layers. bf16 storage: an output is rounded once (at most
2^-8 relative) and computed from at most two operands that were rounded as
matrix operands (2^-8 each), so 3 * 2^-8 = 1.2e-2 bounds both norms; fp32
results of bf16 inputs (states, dw) see no output rounding: 2^-7. Sums are
exact enough in fp32 not to matter beside that."""
import numpy as np
import pytest

from conftest import rel_err, rel_max
from oracle import sequence as orc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = {"f32": 1e-5, "bf16": 3 * 2.0 ** -8}
TOL32 = {"f32": 1e-5, "bf16": 2.0 ** -7}  # fp32 results
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


def _check(name, got, want, tol, terms=None):
    """want is rounded to fp32 first: below fp32's range it is 0. terms: what `want` is a difference of, where its
    error follows their size."""
    got, want = _np(got) if isinstance(got, torch.Tensor) else got, np.asarray(want, np.float32).astype(np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    if terms is None:
        e, m = rel_err(got, want), rel_max(got, want)
    else:
        e, m = (rel(terms + (got - want), terms) for rel in (rel_err, rel_max))
    assert e <= tol and m <= tol, (name, e, m)


def _rand(rng, *shape, dtype="f32"):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DT[dtype]).cuda()


def _qkv(rng, T, heads, kv, dk, dv, dtype, layout):
    """contiguous tensors, views of one projection (fused), or such views off the 16-byte grid (odd)."""
    if layout == "contiguous":
        return _rand(rng, T, heads, dk, dtype=dtype), _rand(rng, T, kv, dk, dtype=dtype), _rand(rng, T, kv, dv, dtype=dtype)
    pad = 3 if layout == "odd" else 0
    a = _rand(rng, T, pad + (heads + kv) * dk + kv * dv, dtype=dtype)[:, pad:]
    return (a[:, :heads * dk].unflatten(1, (heads, dk)), a[:, heads * dk:(heads + kv) * dk].unflatten(1, (kv, dk)),
            a[:, (heads + kv) * dk:].unflatten(1, (kv, dv)))


def _rates(rng, heads):
    return torch.from_numpy(rng.uniform(0.0, 0.3, heads).astype(np.float32) ** 2).cuda()


ATTENTION = [
    # lengths, heads, kv_heads, dk, dv, dtype, layout
    ([1], 1, 1, 1, 1, "f32", "contiguous"),
    ([0], 2, 1, 16, 16, "bf16", "contiguous"),
    ([0, 5, 0, 1, 33, 0], 4, 4, 16, 16, "f32", "contiguous"),
    ([31, 32, 33, 64, 65], 4, 2, 32, 32, "f32", "fused"),
    ([31, 32, 33, 64, 65], 4, 2, 32, 32, "bf16", "fused"),
    ([63, 1, 129, 2, 300], 2, 2, 64, 64, "bf16", "fused"),
    ([63, 1, 129, 2, 300], 2, 2, 64, 64, "f32", "odd"),
    ([17, 96, 200], 3, 1, 128, 128, "bf16", "odd"),
    ([17, 96, 200], 3, 1, 128, 128, "f32", "fused"),
    ([40, 7, 77], 6, 3, 5, 7, "f32", "odd"),
    ([40, 7, 77], 6, 3, 5, 7, "bf16", "odd"),
    ([50, 81], 2, 1, 100, 20, "bf16", "fused"),
    ([50, 81], 2, 1, 24, 128, "f32", "contiguous"),
    ([50, 81], 2, 2, 128, 8, "bf16", "contiguous"),
    ([1500], 1, 1, 64, 64, "f32", "contiguous"),
    ([2111], 2, 1, 32, 48, "bf16", "fused"),
    ([900, 3, 1201], 2, 2, 128, 128, "bf16", "contiguous"),
]


@pytest.mark.parametrize("lengths,heads,kv,dk,dv,dtype,layout", ATTENTION)
def test_attention(lengths, heads, kv, dk, dv, dtype, layout):
    """o, final states and the gradients of q, k, v and the initial states, with and without states."""
    rng = np.random.default_rng(sum(lengths) * 131 + dk * 7 + dv)
    T, n = sum(lengths), len(lengths)
    print(f"case: attention {lengths} heads {heads}/{kv} dims {dk}x{dv} {dtype} {layout}", flush=True)
    q, k, v = _qkv(rng, T, heads, kv, dk, dv, dtype, layout)
    do = _rand(rng, T, heads, dv, dtype=dtype)
    a = _rates(rng, heads)
    op = _seq().DecayAttention(lengths, heads, dk, dv, a, dtype=DT[dtype], kv_heads=kv)
    scale, tol = dk ** -0.5, TOL[dtype]
    nq, nk, nv, ndo, na = _np(q), _np(k), _np(v), _np(do), _np(a)
    o = op.forward(q, k, v).clone()
    grads = [g.clone() for g in op.backward(do)]
    wo, _ = orc.attention_forward(nq, nk, nv, lengths, na, scale)
    want = orc.attention_backward(nq, nk, nv, lengths, na, scale, ndo)
    _check("o", o, wo, tol)
    for name, g, w in zip(("dq", "dk", "dv"), grads, want):
        _check(name, g, w, tol)
    st, ds = _rand(rng, n, heads, dk, dv), _rand(rng, n, heads, dk, dv)
    o, final = op.forward(q, k, v, state=st, final_state=True)
    got = op.backward(do, dstate=ds)
    wo, wf = orc.attention_forward(nq, nk, nv, lengths, na, scale, _np(st))
    want = orc.attention_backward(nq, nk, nv, lengths, na, scale, ndo, _np(st), _np(ds))
    _check("o", o, wo, tol)
    _check("final", final, wf, TOL32[dtype])
    for name, g, w in zip(("dq", "dk", "dv", "dstate"), got, want):
        _check(name, g, w, TOL32[dtype] if name == "dstate" else tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_extreme_rates(dtype):
    """No decay, a decay that leaves nothing of the token before (rates of 200 and infinity), and one in between."""
    rng = np.random.default_rng(5)
    lengths, heads, d = [70, 130], 4, 32
    q, k, v = _qkv(rng, 200, heads, heads, d, d, dtype, "contiguous")
    do, st = _rand(rng, 200, heads, d, dtype=dtype), _rand(rng, 2, heads, d, d)
    a = torch.tensor([0.0, 200.0, float("inf"), 2.0], device="cuda")
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype], scale=1.0)
    o, final = op.forward(q, k, v, state=st, final_state=True)
    got = op.backward(do, dstate=st)
    na = np.array([0.0, 200.0, 1e6, 2.0])
    wo, wf = orc.attention_forward(_np(q), _np(k), _np(v), lengths, na, 1.0, _np(st))
    want = orc.attention_backward(_np(q), _np(k), _np(v), lengths, na, 1.0, _np(do), _np(st), _np(st))
    for h in range(heads):  # each head by itself: their sizes differ
        _check(f"o[{h}]", o[:, h], wo[:, h], TOL[dtype])
        _check(f"final[{h}]", final[:, h], wf[:, h], TOL32[dtype])
        for name, g, w in zip(("dq", "dk", "dv"), got, want):
            _check(f"{name}[{h}]", g[:, h], w[:, h], TOL[dtype])
        _check(f"dstate[{h}]", got[3][:, h], want[3][:, h], TOL32[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_keeps_nan_in_its_example(dtype):
    """A NaN or infinite token reaches the later tokens of its own example and head, nothing else: earlier tokens and
    other examples keep their bits."""
    rng = np.random.default_rng(6)
    lengths, heads, d = [45, 100, 37], 2, 64
    q, k, v = _qkv(rng, 182, heads, heads, d, d, dtype, "contiguous")
    do = _rand(rng, 182, heads, d, dtype=dtype)
    a = _rates(rng, heads)
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    o = op.forward(q, k, v).clone()
    dq, dk, dv = (g.clone() for g in op.backward(do))
    for bad in (float("nan"), float("inf")):
        k2 = k.clone()
        k2[45 + 50, 0, 3] = bad  # token 50 of the second example, head 0
        o2 = op.forward(q, k2, v).clone()
        dq2, dk2, dv2 = (g.clone() for g in op.backward(do))
        for x, y in ((o, o2), (dq, dq2)):
            assert torch.equal(x[:45], y[:45]) and torch.equal(x[145:], y[145:]) and torch.equal(x[:, 1], y[:, 1])
            assert torch.equal(x[45:64, 0], y[45:64, 0])  # well before it
        assert torch.equal(o[45:95, 0], o2[45:95, 0]), "an earlier token sees a later one"
        assert not torch.isfinite(o2[95:145, 0]).all(1).any()
        assert torch.equal(dv[:45], dv2[:45]) and torch.equal(dv[145:], dv2[145:]) and torch.equal(dv[:, 1], dv2[:, 1])
        assert not torch.isfinite(dv2[95, 0]).all()


@pytest.mark.parametrize("dtype,d", [("f32", 16), ("f32", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_keeps_earlier_tokens_from_a_later_nan_value(dtype, d):
    """A value that is not finite reaches its own column of the outputs, from its token on; as a key it is a value of
    dq's scan, as a gradient of o one of dv's, which runs from the end."""
    rng = np.random.default_rng(16)
    lengths, heads, at = [45, 100], 2, 45 + 40
    q, k, v = _qkv(rng, 145, heads, heads, d, d, dtype, "contiguous")
    do, a = _rand(rng, 145, heads, d, dtype=dtype), _rates(rng, heads)
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    o = op.forward(q, k, v).clone()
    dq, dk, dv = (g.clone() for g in op.backward(do))
    for bad in (float("nan"), float("inf"), -float("inf")):
        v2, k2, do2 = v.clone(), k.clone(), do.clone()
        for t in (v2, k2, do2):
            t[at, 1, 5] = bad
        o2 = op.forward(q, k, v2)
        others = [c for c in range(d) if c != 5]
        _check("before", o2[:at], _np(o[:at]), TOL[dtype])
        _check("other columns", o2[:, :, others], _np(o[:, :, others]), TOL[dtype])
        assert not torch.isfinite(o2[at:, 1, 5]).any()
        op.forward(q, k2, v)
        dq2 = op.backward(do)[0]
        _check("before", dq2[:at], _np(dq[:at]), TOL[dtype])
        _check("other columns", dq2[:, :, others], _np(dq[:, :, others]), TOL[dtype])
        assert not torch.isfinite(dq2[at:, 1, 5]).any()
        op.forward(q, k, v)
        dv2 = op.backward(do2)[2]
        _check("after", dv2[at + 1:], _np(dv[at + 1:]), TOL[dtype])
        _check("other columns", dv2[:, :, others], _np(dv[:, :, others]), TOL[dtype])
        assert not torch.isfinite(dv2[45:at + 1, 1, 5]).any()


@pytest.mark.parametrize("dtype,dim", [("f32", 16), ("bf16", 128)])
def test_attention_does_not_depend_on_its_neighbours(dtype, dim):
    """Examples packed together against each alone: the same up to the order of sums; twice the same call: the same bits."""
    rng = np.random.default_rng(7)
    lengths, heads = [100, 260, 31], 2
    q, k, v = _qkv(rng, 391, heads, 1, dim, dim, dtype, "fused")
    do, a = _rand(rng, 391, heads, dim, dtype=dtype), _rates(rng, heads)
    new = lambda n: _seq().DecayAttention(n, heads, dim, dim, a, dtype=DT[dtype], kv_heads=1)  # noqa: E731
    op = new(lengths)
    first = [op.forward(q, k, v).clone()] + [g.clone() for g in op.backward(do)]
    again = [op.forward(q, k, v).clone()] + [g.clone() for g in op.backward(do)]
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    t = 0
    for n in lengths:
        s = slice(t, t + n)
        one = new([n])
        alone = [one.forward(q[s], k[s], v[s])] + list(one.backward(do[s]))
        for x, y in zip(first, alone):
            _check("alone", x[s], _np(y), TOL[dtype])
        t += n


@pytest.mark.parametrize("dtype,d,heads,n", [("f32", 16, 8, 9000), ("bf16", 64, 2, 40), ("bf16", 128, 4, 3)])
def test_attention_one_long_among_short(dtype, d, heads, n):
    """One long example among short and empty ones, which segments are made for; the long one in the middle, its
    states in and out."""
    rng = np.random.default_rng(n)
    lengths = rng.integers(0, 3, n)
    lengths[n // 2] = 3333
    T = int(lengths.sum())
    print(f"case: {n} examples, one of 3333 tokens, {heads} heads of {d}, {dtype}", flush=True)
    q, k, v = _qkv(rng, T, heads, heads, d, d, dtype, "fused")
    do, a = _rand(rng, T, heads, d, dtype=dtype), _rates(rng, heads)
    st, ds = _rand(rng, n, heads, d, d), _rand(rng, n, heads, d, d)
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype])
    o, final = op.forward(q, k, v, state=st, final_state=True)
    got = op.backward(do, dstate=ds)
    some = slice(n // 2 - 1, n // 2 + 2)  # the oracle walks three examples
    t0 = int(lengths[:n // 2 - 1].sum())
    t = slice(t0, t0 + int(lengths[some].sum()))
    cut = lambda x: _np(x[t])  # noqa: E731
    args = cut(q), cut(k), cut(v), lengths[some], _np(a), d ** -0.5
    wo, wf = orc.attention_forward(*args, _np(st[some]))
    want = orc.attention_backward(*args, cut(do), _np(st[some]), _np(ds[some]))
    _check("o", o[t], wo, TOL[dtype])
    _check("final", final[some], wf, TOL32[dtype])
    for name, g, w in zip(("dq", "dk", "dv"), got, want):
        _check(name, g[t], w, TOL[dtype])
    _check("dstate", got[3][some], want[3], TOL32[dtype])
    empty = torch.from_numpy(lengths == 0).cuda()
    assert torch.equal(final[empty], st[empty]) and torch.equal(got[3][empty], ds[empty])


def test_attention_gradient_by_differences():
    """o is linear in q, k and v each, so a difference quotient with a step of 1 is exact up to rounding."""
    rng = np.random.default_rng(8)
    lengths, heads, d = [33, 190], 2, 32
    q, k, v = _qkv(rng, 223, heads, 1, d, d, "f32", "contiguous")
    do, st, a = _rand(rng, 223, heads, d), _rand(rng, 2, heads, d, d), _rates(rng, heads)
    op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=torch.float32, kv_heads=1)
    loss = lambda q, k, v, st: (op.forward(q, k, v, state=st).double() * do.double()).sum()  # noqa: E731
    op.forward(q, k, v, state=st)
    grads = [g.clone() for g in op.backward(do)]
    args = [q, k, v, st]
    for i, g in enumerate(grads):
        d_ = _rand(rng, *g.shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + d_, args[i] - d_
        num, got = float(loss(*up) - loss(*down)) / 2, float((g.double() * d_.double()).sum())
        size = float(g.double().norm() * d_.double().norm())
        assert abs(num - got) <= 1e-5 * size, (i, num, got)


def test_attention_cuts_wrong_offsets():
    """Offsets beyond the tensors or not ascending: tokens outside stay as they were, nothing is read there."""
    import ctypes

    from paper_1902_11208_amd import _lib

    rng = np.random.default_rng(9)
    T, heads, d = 50, 2, 32
    q, k, v = _qkv(rng, T, heads, heads, d, d, "f32", "contiguous")
    a = _rates(rng, heads)
    L = _lib.lib()
    desc = _lib.AttentionDesc(heads, heads, d, d, 0, 1.0)
    view = lambda t: _lib.Heads(t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
    for offsets, rows in (([0, 1 << 40, 1 << 41], slice(0, 50)), ([-5, 20, 10], slice(0, 20)), ([60, 70, 80], slice(0, 0)),
                          ([0, 45, 50], slice(0, 50)), ([50, 0, 50], slice(0, 50))):
        off = torch.tensor(offsets, device="cuda")
        buf = torch.full((T + 64, heads, d), 7.0, device="cuda")
        ws = torch.empty(int(L.mdlstm_attention_workspace_bytes(ctypes.byref(desc), 2, T, 50, 0)), dtype=torch.uint8,
                         device="cuda")
        _lib.check(L.mdlstm_attention_forward(desc, 2, T, 50, off.data_ptr(), None, a.data_ptr(), view(q), view(k), view(v),
                                              None, buf.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                              torch.cuda.current_stream().cuda_stream))
        torch.cuda.synchronize()
        assert bool((buf[rows.stop:] == 7.0).all()), offsets
        assert not bool((buf[rows] == 7.0).any()), offsets
    # an order that is no permutation: entries outside are skipped, an example not listed stays as it was
    off, order = torch.tensor([0, 20, 50], device="cuda"), torch.tensor([7, 1], dtype=torch.int32, device="cuda")
    buf = torch.full((T, heads, d), 7.0, device="cuda")
    _lib.check(L.mdlstm_attention_forward(desc, 2, T, 50, off.data_ptr(), order.data_ptr(), a.data_ptr(), view(q), view(k),
                                          view(v), None, buf.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                          torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert bool((buf[:20] == 7.0).all()) and not bool((buf[20:] == 7.0).any())
    # in segments: offsets that descend, with the long example's length given as the longest
    T = 2000
    q, k, v = _qkv(rng, T, heads, heads, d, d, "f32", "contiguous")
    for offsets in ([0, 1500, 300, 2000], [2000, 0, 1 << 50, -7], [1900, 100, 1000, 1], [0, 0, 0, 0]):
        buf = torch.full((T + 64, heads, d), 7.0, device="cuda")
        ws = torch.empty(int(L.mdlstm_attention_workspace_bytes(ctypes.byref(desc), 3, T, T, 0)), dtype=torch.uint8,
                         device="cuda")
        assert ws.numel() > 1 << 16  # segments
        off = torch.tensor(offsets, device="cuda")
        _lib.check(L.mdlstm_attention_forward(desc, 3, T, T, off.data_ptr(), None, a.data_ptr(), view(q), view(k), view(v),
                                              None, buf.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                              torch.cuda.current_stream().cuda_stream))
        torch.cuda.synchronize()
        assert bool((buf[T:] == 7.0).all()), offsets


@pytest.mark.parametrize("heads,kv,dk,dv,dtype,layout,n", [
    (1, 1, 1, 1, "f32", "contiguous", 1), (4, 4, 32, 32, "f32", "contiguous", 3), (8, 2, 64, 64, "bf16", "fused", 9),
    (4, 1, 128, 128, "bf16", "fused", 5), (6, 3, 5, 7, "f32", "odd", 4), (2, 2, 100, 20, "bf16", "odd", 33),
    (2, 1, 20, 100, "f32", "fused", 1), (16, 4, 128, 128, "f32", "contiguous", 70)])
def test_step(heads, kv, dk, dv, dtype, layout, n):
    """Rows in scattered slots, idle rows (slots below and beyond the states), untouched states keep their bits."""
    rng = np.random.default_rng(n * 31 + dk)
    print(f"case: step {n} rows heads {heads}/{kv} dims {dk}x{dv} {dtype} {layout}", flush=True)
    q, k, v = _qkv(rng, n, heads, kv, dk, dv, dtype, layout)
    a, slots = _rates(rng, heads), n + 3
    st = _rand(rng, slots, heads, dk, dv)
    at = rng.permutation(slots)[:n].astype(np.int32)
    if n > 2:
        at[0], at[1] = -1, slots
    before = st.clone()
    o = _seq().decay_attention_step(q, k, v, st, a, slots=torch.from_numpy(at).cuda())
    wo, ws = orc.attention_step(_np(q), _np(k), _np(v), _np(before), _np(a), at, dk ** -0.5)
    _check("o", o, wo, TOL[dtype])
    _check("state", st, ws, 1e-5)
    idle = [s for s in range(slots) if s not in at]
    assert torch.equal(st[idle], before[idle])
    # without slots: row i advances state i
    st2 = before.clone()
    o2 = _seq().decay_attention_step(q, k, v, st2, a, out=torch.empty_like(o))
    wo, ws = orc.attention_step(_np(q), _np(k), _np(v), _np(before), _np(a), np.arange(n), dk ** -0.5)
    _check("o", o2, wo, TOL[dtype])
    _check("state", st2, ws, 1e-5)


def test_steps_follow_a_prompt():
    """A prompt through the packed form, then token by token: the same as the whole sequence at once."""
    rng = np.random.default_rng(11)
    heads, d, n, m = 4, 32, 90, 6
    q, k, v = _qkv(rng, 2 * (n + m), heads, heads, d, d, "f32", "contiguous")
    a = _rates(rng, heads)
    whole, final = _seq().DecayAttention([n + m] * 2, heads, d, d, a, dtype=torch.float32).forward(q, k, v, final_state=True)
    first = [torch.cat([t[:n], t[n + m:2 * n + m]]) for t in (q, k, v)]
    _, st = _seq().DecayAttention([n, n], heads, d, d, a, dtype=torch.float32).forward(*first, final_state=True)
    for i in range(m):
        at = [n + i, 2 * n + m + i]
        o = _seq().decay_attention_step(q[at], k[at], v[at], st, a)
        _check("o", o, _np(whole[at]), 1e-5)
    _check("state", st, _np(final), 1e-5)


def test_binding_refuses_wrong_tensors():
    """Shapes, types, devices and layouts that the kernels would misread."""
    sq = _seq()
    op = sq.DecayAttention([3, 4], 4, 8, 6, torch.zeros(4, device="cuda"), dtype=torch.float32, kv_heads=2)
    q, k, v = (torch.zeros(7, h, d, device="cuda") for h, d in ((4, 8), (2, 8), (2, 6)))
    st = torch.zeros(2, 4, 8, 6, device="cuda")
    with pytest.raises(ValueError, match="forward call"):
        op.backward(torch.zeros(7, 4, 6, device="cuda"))
    for a, says in (((q[:6], k, v), "q has shape"), ((q, q, v), "k has shape"), ((q, k, k), "v has shape"),
                    ((q.bfloat16(), k, v), "q has dtype"), ((q.cpu(), k, v), "q is on"),
                    ((torch.zeros(7, 4, 16, device="cuda")[:, :, ::2], k, v), "last dimension")):
        with pytest.raises(ValueError, match=says):
            op.forward(*a)
    with pytest.raises(ValueError, match="state has shape"):
        op.forward(q, k, v, state=st[:1])
    with pytest.raises(ValueError, match="state must be contiguous"):
        op.forward(q, k, v, state=torch.zeros(2, 4, 6, 8, device="cuda").transpose(2, 3))
    op.forward(q, k, v, state=st)
    with pytest.raises(ValueError, match="do has shape"):
        op.backward(q)
    with pytest.raises(ValueError, match="dstate has dtype"):
        op.backward(torch.zeros(7, 4, 6, device="cuda"), dstate=st.double())
    norm = sq.ResidualNorm(torch.ones(8, device="cuda"), 5, dtype=torch.float32)
    x = torch.zeros(5, 8, device="cuda")
    with pytest.raises(ValueError, match="forward call"):
        norm.backward(x)
    for t, r, says in ((x[:4], None, "x has shape"), (x.bfloat16(), None, "x has dtype"), (x, x.cpu(), "residual is on"),
                       (torch.zeros(8, 5, device="cuda").t(), None, "contiguous along its rows"),
                       (x[:1].expand(5, 8), None, "overlap")):
        with pytest.raises(ValueError, match=says):
            norm.forward(t, r)
    norm.forward(x)
    with pytest.raises(ValueError, match="dy must be contiguous"):
        norm.backward(torch.zeros(5, 16, device="cuda")[:, :8])
    with pytest.raises(ValueError, match="not a 64-bit"):
        norm.forward(x, seed=-1)
    from paper_1902_11208_amd import MdlstmError

    with pytest.raises(MdlstmError, match="probability"):  # what the library refuses
        sq.dropout(x, 1.5, 0)
    with pytest.raises(ValueError, match="at most 128"):
        sq.DecayAttention([3], 4, 200, 6, torch.zeros(4, device="cuda"))


# --- norm and dropout ----------------------------------------------------------
def _strided(rng, rows, cols, dtype, layout):
    if layout == "contiguous":
        return _rand(rng, rows, cols, dtype=dtype)
    return _rand(rng, rows, cols + (16 if layout == "wide" else 3), dtype=dtype)[:, (8 if layout == "wide" else 2):][:, :cols]


NORM = [
    # rows, cols, dtype, p, residual, layout
    (1, 1, "f32", 0.0, False, "contiguous"),
    (5, 3, "f32", 0.5, True, "odd"),
    (7, 64, "f32", 0.25, True, "contiguous"),
    (9, 64, "bf16", 0.0, False, "wide"),
    (33, 127, "bf16", 0.1, True, "contiguous"),
    (4, 256, "f32", 0.0, True, "wide"),
    (3, 500, "bf16", 0.3, False, "contiguous"),
    (130, 512, "bf16", 0.1, True, "wide"),
    (2, 1000, "f32", 0.2, True, "contiguous"),
    (3, 2048, "bf16", 0.1, True, "contiguous"),
    (2, 4095, "f32", 0.0, True, "odd"),
    (2, 5000, "bf16", 0.1, True, "contiguous"),
    (1, 16384, "bf16", 0.0, True, "contiguous"),
    (2, 20001, "f32", 0.1, False, "contiguous"),
    (1, 32768, "f32", 0.0, False, "contiguous"),
    (3000, 40, "f32", 0.0, True, "contiguous"),
]


def _factor(rows, cols, p, seed, call):
    return orc.dropout_scale(rows * cols, p, seed, call).reshape(rows, cols) if p else None


@pytest.mark.parametrize("rows,cols,dtype,p,residual,layout", NORM)
def test_norm(rows, cols, dtype, p, residual, layout):
    rng = np.random.default_rng(rows * 7 + cols)
    print(f"case: norm {rows}x{cols} {dtype} p {p} residual {residual} {layout}", flush=True)
    x = _strided(rng, rows, cols, dtype, layout)
    r = _strided(rng, rows, cols, dtype, layout) if residual else None
    w = 1 + 0.3 * _rand(rng, cols)
    dy, dh = _rand(rng, rows, cols, dtype=dtype), _rand(rng, rows, cols, dtype=dtype)
    op = _seq().ResidualNorm(w, rows, dtype=DT[dtype], eps=1e-5, dropout=p)
    y, h = op.forward(x, r, seed=(5 << 40) + 3, call=(1 << 33) + 2)
    f = _factor(rows, cols, p, (5 << 40) + 3, (1 << 33) + 2)
    wy, wh, _ = orc.norm_forward(_np(x), _np(w), 1e-5, None if r is None else _np(r), f)
    _check("y", y, wy, TOL[dtype])
    _check("h", h, wh, TOL[dtype])
    if f is not None and r is None:
        assert np.array_equal(_np(h) == 0, wh == 0)
    for g in (dh, None):
        dx, dres, dw = op.backward(dy, g)
        wx, wr, ww = orc.norm_backward(_np(h), _np(w), 1e-5, _np(dy), None if g is None else _np(g), f)
        # rstd (g - c mean(g c)): with a single column all of it cancels but eps / h^2
        rstd = 1 / np.sqrt((_np(h) ** 2).mean(1, keepdims=True) + 1e-5)
        terms = rstd * _np(dy) * _np(w) + (0 if g is None else _np(g))
        _check("dx", dx, wx, TOL[dtype], terms)
        _check("dw", dw, ww, TOL32[dtype])
        assert (dres is None) == (r is None)
        if r is not None:
            _check("dresidual", dres, wr, TOL[dtype])
        if f is not None:
            assert bool((dx[torch.from_numpy(f == 0).cuda()] == 0).all())


@pytest.mark.parametrize("rows,cols,dtype,residual,layout", [
    (1, 1, "f32", False, "contiguous"), (6, 100, "bf16", True, "odd"), (5, 64, "f32", True, "contiguous"),
    (3, 4096, "bf16", True, "contiguous"), (2, 5000, "bf16", False, "wide"), (40, 1024, "bf16", True, "contiguous")])
def test_norm_fp8(rows, cols, dtype, residual, layout):
    """Scale max|y| / 448 per row; each value within half a step of e4m3: 2^-4 of it, or 2^-10 below the normal range,
    and 1e-5 of the row's scale for the rounding of y itself."""
    rng = np.random.default_rng(rows + cols)
    x = _strided(rng, rows, cols, dtype, layout)
    r = _strided(rng, rows, cols, dtype, layout) if residual else None
    w = 1 + 0.3 * _rand(rng, cols)
    op = _seq().ResidualNorm(w, rows, dtype=DT[dtype], eps=1e-5, out="fp8")
    y, s, h = op.forward(x, r)
    wy, wh, _ = orc.norm_forward(_np(x), _np(w), 1e-5, None if r is None else _np(r))
    _check("scale", s, np.abs(wy).max(1) / 448, 1e-5)
    _check("h", h, wh, TOL[dtype])
    q, want = _np(y.float()), wy / _np(s)[:, None]
    assert np.all(np.abs(q - want) <= np.maximum(np.abs(want) * 2.0 ** -4, 2.0 ** -10) + 1e-5 * 448)
    assert np.all(np.abs(q).max(1) == 448)


def test_norm_rows_that_are_zero_or_not_finite():
    """Rows of zeros, with an infinity, with a NaN, and of the smallest values, beside an ordinary one, which keeps its bits."""
    rng = np.random.default_rng(13)
    x = _rand(rng, 5, 192)
    clean = x.clone()
    x[0] = 0
    x[1, 7] = float("inf")
    x[2, 100] = float("nan")
    x[3] = 1e-38
    w = 1 + 0.1 * _rand(rng, 192)
    for rows in (x, clean):
        op = _seq().ResidualNorm(w, 5, dtype=torch.float32)
        op8 = _seq().ResidualNorm(w, 5, dtype=torch.float32, out="fp8")
        y, _ = op.forward(rows)
        y8, s, _ = op8.forward(rows)
        if rows is x:
            got, got8, gots = y.clone(), y8.clone(), s.clone()
    assert torch.equal(got[4], y[4]) and torch.equal(got8[4].view(torch.uint8), y8[4].view(torch.uint8)) and gots[4] == s[4]
    assert not got[0].any() and not got8[0].float().any() and gots[0] == 2.0 ** -126
    assert torch.isnan(got[1, 7]) and not got[1, :7].any() and torch.isnan(gots[1])
    assert torch.isnan(got[2]).all() and torch.isnan(gots[2]) and torch.isnan(got8[2].float()).all()
    assert torch.isfinite(got[3]).all() and torch.isfinite(got8[3].float()).all()


@pytest.mark.parametrize("shape,dtype,p,residual,layout", [
    ((1,), "f32", 0.5, False, "contiguous"), ((7, 9), "f32", 0.3, True, "contiguous"), ((3, 5, 11), "bf16", 0.1, True, "contiguous"),
    ((40, 64), "bf16", 0.9, False, "wide"), ((40, 61), "f32", 0.2, True, "odd"), ((1000, 33), "bf16", 0.5, False, "contiguous"),
    ((0, 8), "f32", 0.5, False, "contiguous"), ((13, 8), "f32", 0.0, True, "contiguous"), ((13, 8), "f32", 1.0, True, "contiguous"),
    ((13, 8), "f32", 1e-7, False, "contiguous")])
def test_dropout(shape, dtype, p, residual, layout):
    rng = np.random.default_rng(17)
    mk = lambda: _rand(rng, *shape, dtype=dtype) if layout == "contiguous" else _strided(rng, *shape, dtype, layout)  # noqa: E731
    x, r = mk(), mk() if residual else None
    seed, call = 0xFEDCBA9876543210, 0x123456789ABCDEF0
    y = _seq().dropout(x, p, seed, call, residual=r)
    f = orc.dropout_scale(x.numel(), p, seed, call).reshape(shape)
    want = _np(x) * f + (0 if r is None else _np(r))
    _check("y", y, want, TOL[dtype])
    if r is None:
        assert np.array_equal(_np(y) == 0, want == 0)
        # a dropped element is zero whatever it held
        bad = torch.full_like(x, float("nan"))
        assert np.array_equal(np.isnan(_np(_seq().dropout(bad, p, seed, call))), f != 0)
    if layout == "contiguous":  # in place, and off the 16-byte grid: the same bits
        z = x.clone()
        assert torch.equal(_seq().dropout(z, p, seed, call, residual=r, out=z), y) and z.numel() == x.numel()
        off = torch.empty(x.numel() + 3, dtype=DT[dtype], device="cuda")[3:].view(shape)
        off.copy_(x)
        assert torch.equal(_seq().dropout(off, p, seed, call, residual=r), y)


def test_dropout_streams_differ():
    """Another seed or call is another mask; 16-bit halves of one block are not each other's copies."""
    x = torch.ones(1 << 16, device="cuda")
    ys = [_seq().dropout(x, 0.5, s, c) != 0 for s, c in ((1, 1), (1, 2), (2, 1), (1 + (1 << 32), 1), (1, 1 + (1 << 32)))]
    n = x.numel()
    for i in range(len(ys)):
        assert abs(int(ys[i].sum()) - n // 2) < 5 * (n ** 0.5) / 2
        for j in range(i):
            assert abs(int((ys[i] ^ ys[j]).sum()) - n // 2) < 5 * (n ** 0.5) / 2, (i, j)
    b = ys[0].view(-1, 8)
    for i in range(8):
        for j in range(i):
            assert abs(int((b[:, i] ^ b[:, j]).sum()) - n // 16) < 5 * ((n // 8) ** 0.5) / 2, (i, j)


def test_other_stream_and_graph():
    """The calls on a side stream, and replayed from a graph with eager work between the replays: the same bits."""
    rng = np.random.default_rng(19)
    lengths, heads, d = [300, 0, 45], 2, 64
    q, k, v = _qkv(rng, 345, heads, 1, d, d, "bf16", "contiguous")
    do, a = _rand(rng, 345, heads, d, dtype="bf16"), _rates(rng, heads)
    op = _seq().DecayAttention(lengths, heads, d, d, a, kv_heads=1)
    x, res = _rand(rng, 345, 128, dtype="bf16"), _rand(rng, 345, 128, dtype="bf16")
    norm = _seq().ResidualNorm(torch.ones(128, device="cuda"), 345, dropout=0.2)
    out = torch.empty_like(x)

    def step():
        y, h = norm.forward(x, res, seed=3, call=4)
        return [op.forward(q, k, v), *op.backward(do), y, h, *norm.backward(y, h), _seq().dropout(x, 0.3, 5, 6, out=out)]

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [t.clone() for t in step()]
    s.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
        _ = (x.float() @ x.float().t()).sum().item()


def test_poisoned_workspaces_change_nothing(monkeypatch):
    """With MDLSTM_POISON_WORKSPACE=1 the workspaces are NaN at the start of a call: the same bits come out."""
    rng = np.random.default_rng(23)
    for lengths, heads, kv, d, dtype in (([3000, 1, 0], 2, 2, 32, "f32"), ([2500], 4, 2, 64, "bf16"), ([70, 9], 4, 1, 16, "f32")):
        T = sum(lengths)
        q, k, v = _qkv(rng, T, heads, kv, d, d, dtype, "contiguous")
        do, a, st = _rand(rng, T, heads, d, dtype=dtype), _rates(rng, heads), _rand(rng, len(lengths), heads, d, d)
        op = _seq().DecayAttention(lengths, heads, d, d, a, dtype=DT[dtype], kv_heads=kv)
        norm = _seq().ResidualNorm(torch.ones(heads * d, device="cuda"), T, dtype=DT[dtype])
        x, dy = _rand(rng, T, heads * d, dtype=dtype), _rand(rng, T, heads * d, dtype=dtype)

        def run():
            norm.forward(x)
            return [t.clone() for t in (*op.forward(q, k, v, state=st, final_state=True), *op.backward(do, dstate=st),
                                        norm.backward(dy)[0], norm.backward(dy)[2])]

        want = run()
        monkeypatch.setenv("MDLSTM_POISON_WORKSPACE", "1")
        got = run()
        monkeypatch.delenv("MDLSTM_POISON_WORKSPACE")
        assert all(torch.equal(g, w) for g, w in zip(got, want))
