"""The sequence operators reject bad arguments on the host before any HIP call
(runs without a GPU: FAKE is never dereferenced)."""
import ctypes

import pytest

FAKE = 0x100000
OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 4, 5


@pytest.fixture(scope="module", autouse=True)
def _built(built_lib):
    pass


def _L():
    from paper_1902_11208_amd import _lib

    return _lib


def _desc(heads=4, kv=2, dk=32, dv=16, dtype=0):
    return _L().AttentionDesc(heads, kv, dk, dv, dtype, 1.0)


def _view(p=FAKE, ts=128, hs=32):
    return _L().Heads(p, ts, hs)


ATTENTION_BAD = [
    (dict(desc=None), INVALID), (dict(desc=dict(dtype=2)), INVALID), (dict(desc=dict(heads=0)), INVALID),
    (dict(desc=dict(kv=0)), INVALID), (dict(desc=dict(heads=4, kv=3)), INVALID), (dict(desc=dict(heads=2, kv=4)), INVALID),
    (dict(desc=dict(heads=2048, kv=2048)), UNSUPPORTED), (dict(desc=dict(dk=0)), INVALID), (dict(desc=dict(dv=-1)), INVALID),
    (dict(desc=dict(dk=129)), UNSUPPORTED), (dict(desc=dict(dv=256)), UNSUPPORTED),
    (dict(n=-1), INVALID), (dict(n=1 << 25), INVALID), (dict(tokens=-1), INVALID), (dict(longest=-1), INVALID),
    (dict(longest=101), INVALID), (dict(n=0), INVALID), (dict(tokens=1 << 50, longest=1), INVALID),
    (dict(q=None), INVALID), (dict(q=(0, 128, 32)), INVALID), (dict(k=(FAKE + 2, 128, 32)), INVALID),
    (dict(v=(FAKE, -1, 32)), INVALID), (dict(v=(FAKE, 128, -32)), INVALID), (dict(q=(FAKE, 1 << 62, 32)), INVALID),
    (dict(q=(FAKE, 1 << 58, 1 << 60)), INVALID),
    (dict(order=FAKE + 2), INVALID), (dict(offsets=None), INVALID), (dict(offsets=FAKE + 4), INVALID), (dict(rates=None), INVALID),
    (dict(state=FAKE + 4), INVALID), (dict(out=None), INVALID), (dict(out=FAKE + 8), INVALID), (dict(final=FAKE + 2), INVALID),
    (dict(ws=None), WORKSPACE), (dict(short=1), WORKSPACE), (dict(ws=FAKE + 4), INVALID),
]


@pytest.mark.parametrize("change,code", ATTENTION_BAD)
@pytest.mark.parametrize("backward", [False, True])
def test_attention_errors(change, code, backward):
    L = _L().lib()
    a = dict(desc={}, n=3, tokens=100, longest=50, offsets=FAKE, order=FAKE, rates=FAKE, q=(FAKE, 128, 32), k=(FAKE, 64, 32),
             v=(FAKE, 32, 16), state=None, out=FAKE, final=None, ws=FAKE, short=0)
    a.update(change)
    d = None if a["desc"] is None else _desc(**a["desc"])
    views = [None if a[n] is None else _view(*a[n]) for n in "qkv"]
    need = L.mdlstm_attention_workspace_bytes(d, a["n"], a["tokens"], a["longest"], int(backward))
    size_only = {"desc", "n", "tokens", "longest"}
    assert (need == 0) == (set(change) <= size_only)
    have = max(need, 1 << 20) if not a["short"] else need - 1
    if backward:
        st = L.mdlstm_attention_backward(d, a["n"], a["tokens"], a["longest"], a["offsets"], a["order"], a["rates"], *views,
                                         a["state"], _view(), None, a["out"], FAKE, FAKE, a["final"], a["ws"], have, None)
    else:
        st = L.mdlstm_attention_forward(d, a["n"], a["tokens"], a["longest"], a["offsets"], a["order"], a["rates"], *views,
                                        a["state"], a["out"], a["final"], a["ws"], have, None)
    assert st == code, L.mdlstm_last_error()


def test_attention_of_nothing():
    L = _L().lib()
    d = _desc()
    v = _view(0)
    need = L.mdlstm_attention_workspace_bytes(d, 0, 0, 0, 0)
    assert need >= 16
    assert L.mdlstm_attention_forward(d, 0, 0, 0, None, None, None, v, v, v, None, None, None, FAKE, need, None) == OK
    assert L.mdlstm_attention_step(d, 0, None, v, v, v, None, 0, None, None, None) == OK


@pytest.mark.parametrize("change", [
    dict(n=-1), dict(slots=-1), dict(slots=2), dict(rates=None), dict(state=None), dict(state=FAKE + 4),
    dict(slot=FAKE + 2), dict(out=None), dict(out=FAKE + 4), dict(q=(0, 128, 32)), dict(v=(FAKE + 1, 32, 16))])
def test_step_errors(change):
    L = _L().lib()
    a = dict(n=3, rates=FAKE, q=(FAKE, 128, 32), k=(FAKE, 64, 32), v=(FAKE, 32, 16), state=FAKE, slots=8, slot=None,
             out=FAKE)
    a.update(change)
    st = L.mdlstm_attention_step(_desc(), a["n"], a["rates"], *[_view(*a[n]) for n in "qkv"], a["state"], a["slots"],
                                 a["slot"], a["out"], None)
    assert st == INVALID, L.mdlstm_last_error()


@pytest.mark.parametrize("change", [
    dict(dtype=5), dict(rows=-1), dict(cols=-1), dict(rows=1 << 40, cols=1 << 40), dict(x=None), dict(x=FAKE + 1),
    dict(xs=7), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(r=FAKE, rs=7), dict(r=FAKE + 2), dict(y=None),
    dict(y=FAKE + 2)])
def test_dropout_errors(change):
    L = _L().lib()
    a = dict(dtype=0, rows=4, cols=8, x=FAKE, xs=8, p=0.5, r=None, rs=8, y=FAKE)
    a.update(change)
    assert L.mdlstm_dropout(a["dtype"], a["rows"], a["cols"], a["x"], a["xs"], a["p"], 1, 2, a["r"], a["rs"], a["y"],
                            None) == INVALID
    assert L.mdlstm_dropout(0, 0, 8, None, 8, 0.5, 1, 2, None, 0, None, None) == OK


NORM_BAD = [
    (dict(cols=0), INVALID), (dict(cols=32769), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(eps=float("nan")), INVALID), (dict(p=2.0), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID), (dict(x=None), INVALID), (dict(xs=63), INVALID),
    (dict(r=FAKE, rs=63), INVALID), (dict(w=None), INVALID), (dict(w=FAKE + 2), INVALID)]
NORM_FWD_BAD = NORM_BAD + [
    (dict(y=None), INVALID), (dict(y8=FAKE, scale=FAKE), INVALID), (dict(y=None, y8=FAKE), INVALID),
    (dict(scale=FAKE), INVALID), (dict(h=None, r=FAKE), INVALID), (dict(h=None, p=0.5), INVALID), (dict(h=FAKE + 1), INVALID)]


@pytest.mark.parametrize("change,code", NORM_FWD_BAD)
def test_norm_forward_errors(change, code):
    L = _L()
    a = dict(cols=64, dtype=0, eps=1e-6, p=0.0, rows=5, x=FAKE, xs=64, r=None, rs=64, w=FAKE, h=FAKE, y=FAKE, y8=None,
             scale=None)
    a.update(change)
    d = L.NormDesc(a["cols"], a["dtype"], a["eps"], a["p"])
    assert L.lib().mdlstm_norm_forward(d, a["rows"], a["x"], a["xs"], a["r"], a["rs"], a["w"], 1, 2, a["h"], a["y"],
                                       a["y8"], a["scale"], None, None) == code


@pytest.mark.parametrize("change,code", [c for c in NORM_BAD if "r" not in c[0]] + [
    (dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(dw=None), INVALID), (dict(rstd=None), INVALID),
    (dict(ws=None), WORKSPACE), (dict(short=True), WORKSPACE), (dict(ws=FAKE + 4), INVALID)])
def test_norm_backward_errors(change, code):
    L = _L()
    a = dict(cols=64, dtype=0, eps=1e-6, p=0.0, rows=5, x=FAKE, xs=64, w=FAKE, dy=FAKE, dx=FAKE, dw=FAKE, rstd=FAKE,
             ws=FAKE, short=False)
    a.update(change)
    d = L.NormDesc(a["cols"], a["dtype"], a["eps"], a["p"])
    need = L.lib().mdlstm_norm_workspace_bytes(d, a["rows"])
    have = need - 1 if a["short"] else max(need, 1 << 20)
    assert L.lib().mdlstm_norm_backward(d, a["rows"], a["x"], a["xs"], a["rstd"], a["w"], a["dy"], None, 1, 2, a["dx"], None,
                                        a["dw"], a["ws"], have, None) == code


def test_binding_refusals():
    """Tensors that the C ABI would misread never reach it."""
    torch = pytest.importorskip("torch")
    from paper_1902_11208_amd import sequence

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        sequence.dropout(x, 0.5, 1)  # not on a device
    with pytest.raises(ValueError):
        sequence.ResidualNorm(torch.ones(2, 4), 3)
    with pytest.raises(ValueError):
        sequence.ResidualNorm(torch.ones(8), 3)
    with pytest.raises(ValueError):
        sequence.ResidualNorm(torch.ones(8), 3, out="int8")
    with pytest.raises(ValueError):
        sequence.DecayAttention([1, -1], 2, 4, 4, torch.zeros(2))
    with pytest.raises(ValueError):
        sequence.DecayAttention([1, 1], 2, 4, 4, torch.zeros(2))
    with pytest.raises(TypeError):
        sequence.DecayAttention([1, 1], 2, 4, 4, torch.zeros(2), dtype=torch.float16)
    with pytest.raises(ValueError):
        sequence.decay_attention_step(x, x, x, x, x)
    # the step's and dropout's defects are told before they find no device
    q, st, rates = torch.zeros(5, 4, 8), torch.zeros(9, 4, 8, 6), torch.zeros(4)
    k, v, slots = torch.zeros(5, 2, 8), torch.zeros(5, 2, 6), torch.zeros(5, dtype=torch.int32)
    good = dict(q=q, k=k, v=v, state=st, rates=rates, slots=slots, out=torch.zeros(5, 4, 6))
    wide = torch.zeros(5, 4, 16)
    for change, says in ((dict(), "device"), (dict(q=wide[:, :, :8]), "device"), (dict(q=wide[:, :, ::2]), "last dimension"),
                         (dict(q=torch.zeros(5, 32)), "3 dimensions"), (dict(k=torch.zeros(4, 2, 8)), "k has shape"),
                         (dict(v=v.double()), "v has dtype"), (dict(state=st.transpose(1, 2).contiguous()), "state has shape"),
                         (dict(state=st.bfloat16()), "state has dtype"), (dict(state=st.transpose(0, 1)), "shape"),
                         (dict(rates=torch.zeros(3)), "rates"), (dict(slots=slots.long()), "slots has dtype"),
                         (dict(slots=slots[:3]), "slots has shape"), (dict(out=torch.zeros(5, 4, 12)[:, :, ::2]), "contiguous")):
        a = dict(good, **change)
        with pytest.raises(ValueError, match=says):
            sequence.decay_attention_step(a["q"], a["k"], a["v"], a["state"], a["rates"], slots=a["slots"], out=a["out"])
    with pytest.raises(TypeError):
        sequence.decay_attention_step(q.half(), k.half(), v.half(), st, rates)
    with pytest.raises(TypeError):
        sequence.decay_attention_step(None, k, v, st, rates)
    for t, r, o, says in ((x, x[:3], None, "residual has shape"), (x, x.double(), None, "residual has dtype"),
                          (x, None, torch.zeros(8, 4).t(), "out must be contiguous"), (torch.zeros(4, 16)[:, ::2], None, None, "rows"),
                          (torch.zeros(1, 8).expand(4, 8), None, None, "overlap"), (torch.zeros(2, 3, 4).transpose(0, 1), None, None, "two-dim"),
                          (torch.zeros(4, 20)[:, :8], None, None, "device")):
        with pytest.raises(ValueError, match=says):
            sequence.dropout(t, 0.5, 1, residual=r, out=o)
    with pytest.raises(TypeError):
        sequence.dropout(x.half(), 0.5, 1)
    with pytest.raises(ValueError):
        sequence._u64(-1, "seed")
    with pytest.raises(ValueError):
        sequence._u64(1 << 64, "seed")
