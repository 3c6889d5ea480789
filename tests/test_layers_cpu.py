"""The gated recurrence, the group norm and the loss over a vocabulary reject bad
arguments on the host before any HIP call (runs without a GPU: FAKE is never
dereferenced)."""
import pytest

FAKE = 0x10000000
OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 4, 5


def _at(i):
    """Addresses far from each other, for arguments that must not overlap."""
    return FAKE + (i << 24)


@pytest.fixture(scope="module", autouse=True)
def _built(built_lib):
    pass


def _L():
    from paper_1902_11208_amd import _lib

    return _lib


SEQUENCES_BAD = [(dict(n=-1), INVALID), (dict(n=1 << 25), INVALID), (dict(tokens=-1), INVALID), (dict(longest=-1), INVALID),
                 (dict(longest=101), INVALID), (dict(n=0), INVALID), (dict(tokens=1 << 50, longest=1), INVALID)]
CALL_BAD = [(dict(offsets=None), INVALID), (dict(offsets=FAKE + 4), INVALID), (dict(order=FAKE + 2), INVALID),
            (dict(x=None), INVALID), (dict(x=FAKE + 2), INVALID), (dict(xs=23), INVALID), (dict(xs=(1 << 20) + 1), UNSUPPORTED),
            (dict(xs=1 << 60), INVALID), (dict(ws=None), WORKSPACE), (dict(short=True), WORKSPACE), (dict(ws=_at(9) + 4), INVALID)]
RECURRENCE_BAD = [(dict(desc=None), INVALID), (dict(channels=0), INVALID), (dict(channels=(1 << 20) + 1), UNSUPPORTED),
                  (dict(dtype=2), INVALID), (dict(gate=2), INVALID), (dict(gate=-1), INVALID)] + SEQUENCES_BAD
RECURRENCE_CALL_BAD = CALL_BAD + [(dict(z=None), INVALID), (dict(zs=-1), INVALID), (dict(state=FAKE + 2), INVALID)]
FORWARD_BAD = [(dict(h=None), INVALID), (dict(h=_at(3) + 1), INVALID), (dict(final=FAKE + 2), INVALID), (dict(marks=FAKE + 2), INVALID),
               (dict(h=_at(2)), INVALID), (dict(h=_at(2) + 4 * 99 * 24), INVALID), (dict(final=_at(3)), INVALID),
               (dict(final=_at(8), state=_at(8)), INVALID), (dict(marks=_at(9)), INVALID)]
BACKWARD_BAD = [(dict(g=None), INVALID), (dict(gs=1), INVALID), (dict(marks=None), INVALID), (dict(dz=None), INVALID), (dict(dx=None), INVALID),
                (dict(dz=_at(5)), INVALID), (dict(dz=_at(2)), INVALID), (dict(dstate=_at(8), state=_at(8)), INVALID),
                (dict(dstate=_at(8), dfinal=_at(8)), INVALID), (dict(dfinal=FAKE + 2), INVALID), (dict(dstate=FAKE + 2), INVALID)]


@pytest.mark.parametrize("backward,change,code",
                         [(b, *c) for b in (0, 1) for c in RECURRENCE_BAD + RECURRENCE_CALL_BAD + (BACKWARD_BAD if b else FORWARD_BAD)])
def test_recurrence_errors(backward, change, code):
    M = _L()
    L = M.lib()
    a = dict(desc=1, channels=24, dtype=0, gate=1, n=3, tokens=100, longest=50, offsets=_at(0), order=_at(10), z=_at(1), zs=24, x=_at(2),
             xs=24, state=None, h=_at(3), final=None, marks=_at(4), ws=_at(9), short=False, g=_at(6), gs=24, dfinal=None, dz=_at(3),
             dx=_at(5), dstate=None)
    a.update(change)
    d = M.RecurrenceDesc(a["channels"], a["dtype"], a["gate"]) if a["desc"] else None
    need = L.mdlstm_recurrence_workspace_bytes(d, a["n"], a["tokens"], a["longest"], backward)
    assert (need == 0) == (dict(change) in [c[0] for c in RECURRENCE_BAD])
    have = need - 1 if a["short"] else max(need, 1 << 16)
    head = (d, a["n"], a["tokens"], a["longest"], a["offsets"], a["order"], a["z"], a["zs"], a["x"], a["xs"], a["state"])
    if backward:
        st = L.mdlstm_recurrence_backward(*head, a["marks"], a["g"], a["gs"], a["dfinal"], a["dz"], a["dx"], a["dstate"], a["ws"], have,
                                          None)
    else:
        st = L.mdlstm_recurrence_forward(*head, a["h"], a["final"], a["marks"], a["ws"], have, None)
    assert st == code, L.mdlstm_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(n=-1), INVALID), (dict(slots=-1), INVALID), (dict(slots=2), INVALID), (dict(state=None), INVALID), (dict(state=_at(5) + 2), INVALID),
    (dict(slot=FAKE + 2), INVALID), (dict(h=None), INVALID), (dict(h=_at(1)), INVALID), (dict(h=_at(5)), INVALID), (dict(z=None), INVALID),
    (dict(xs=3), INVALID), (dict(state=_at(2)), INVALID), (dict(gate=7), INVALID), (dict(channels=0), INVALID)])
def test_recurrence_step_errors(change, code):
    M = _L()
    a = dict(channels=8, gate=1, n=3, z=_at(1), zs=8, x=_at(2), xs=8, state=_at(5), slots=8, slot=None, h=_at(6))
    a.update(change)
    st = M.lib().mdlstm_recurrence_step(M.RecurrenceDesc(a["channels"], 0, a["gate"]), a["n"], a["z"], a["zs"], a["x"], a["xs"], a["state"],
                                        a["slots"], a["slot"], a["h"], None)
    assert st == code, M.lib().mdlstm_last_error()


GROUP_BAD = [(dict(desc=None), INVALID), (dict(channels=0), INVALID), (dict(groups=0), INVALID), (dict(groups=5), INVALID),
             (dict(channels=(1 << 20) + 4), UNSUPPORTED), (dict(channels=4097, groups=1), UNSUPPORTED), (dict(dtype=-1), INVALID),
             (dict(act=3), INVALID), (dict(act=-1), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
             (dict(eps=float("inf")), INVALID)] + SEQUENCES_BAD
GROUP_CALL_BAD = CALL_BAD + [(dict(w=None), INVALID), (dict(b=None), INVALID), (dict(w=FAKE + 2), INVALID), (dict(mean=None), INVALID),
                             (dict(rstd=None), INVALID)]
GROUP_FORWARD_BAD = [(dict(y=None), INVALID), (dict(y=_at(2)), INVALID), (dict(y=_at(3) + 2), INVALID), (dict(mean=_at(6)), INVALID)]
GROUP_BACKWARD_BAD = [(dict(dy=None), INVALID), (dict(dys=2), INVALID), (dict(dx=None), INVALID), (dict(dx=_at(2)), INVALID),
                      (dict(dw=None), INVALID), (dict(db=None), INVALID), (dict(dw=_at(12)), INVALID)]


@pytest.mark.parametrize("backward,change,code",
                         [(b, *c) for b in (0, 1) for c in GROUP_BAD + GROUP_CALL_BAD + (GROUP_BACKWARD_BAD if b else GROUP_FORWARD_BAD)])
def test_group_norm_errors(backward, change, code):
    M = _L()
    L = M.lib()
    a = dict(desc=1, channels=24, groups=4, dtype=0, act=2, eps=1e-5, n=3, tokens=100, longest=50, offsets=_at(0), order=_at(10), x=_at(2),
             xs=24, w=_at(7), b=_at(8), y=_at(3), mean=_at(4), rstd=_at(6), dy=_at(5), dys=24, dx=_at(3), dw=_at(11), db=_at(12), ws=_at(9),
             short=False)
    a.update(change)
    d = M.GroupNormDesc(a["channels"], a["groups"], a["dtype"], a["act"], a["eps"]) if a["desc"] else None
    need = L.mdlstm_group_norm_workspace_bytes(d, a["n"], a["tokens"], a["longest"], backward)
    assert (need == 0) == (str(change) in [str(c[0]) for c in GROUP_BAD])
    have = need - 1 if a["short"] else max(need, 1 << 16)
    head = (d, a["n"], a["tokens"], a["longest"], a["offsets"], a["order"], a["x"], a["xs"], a["w"], a["b"])
    if backward:
        st = L.mdlstm_group_norm_backward(*head, a["mean"], a["rstd"], a["dy"], a["dys"], a["dx"], a["dw"], a["db"], a["ws"], have, None)
    else:
        st = L.mdlstm_group_norm_forward(*head, a["y"], a["mean"], a["rstd"], a["ws"], have, None)
    assert st == code, L.mdlstm_last_error()


VOCABULARY_BAD = [(dict(desc=None), INVALID), (dict(dim=0), INVALID), (dict(vocab=0), INVALID), (dict(dim=65537), UNSUPPORTED),
                  (dict(vocab=(1 << 24) + 1), UNSUPPORTED), (dict(dtype=4), INVALID), (dict(rows=-1), INVALID),
                  (dict(rows=(1 << 22) + 1), UNSUPPORTED)]
VOCABULARY_CALL_BAD = [(dict(x=None), INVALID), (dict(x=_at(1) + 1), INVALID), (dict(xs=7), INVALID), (dict(w=None), INVALID),
                       (dict(wstride=7), INVALID), (dict(t=None), INVALID), (dict(t=_at(3) + 4), INVALID), (dict(stats=None), INVALID),
                       (dict(ws=None), WORKSPACE), (dict(short=True), WORKSPACE), (dict(ws=_at(9) + 4), INVALID)]
VOCABULARY_FORWARD_BAD = [(dict(losses=None), INVALID), (dict(losses=_at(5)), INVALID), (dict(stats=_at(1)), INVALID)]
VOCABULARY_BACKWARD_BAD = [(dict(dl=None), INVALID), (dict(dx=None), INVALID), (dict(dw=None), INVALID), (dict(dw=_at(2)), INVALID),
                           (dict(dx=_at(7)), INVALID), (dict(dx=_at(9)), INVALID)]


@pytest.mark.parametrize("backward,change,code", [(b, *c) for b in (0, 1) for c in VOCABULARY_BAD + VOCABULARY_CALL_BAD + (
    VOCABULARY_BACKWARD_BAD if b else VOCABULARY_FORWARD_BAD)])
def test_vocabulary_errors(backward, change, code):
    M = _L()
    L = M.lib()
    a = dict(desc=1, dim=8, vocab=30, dtype=0, rows=5, x=_at(1), xs=8, w=_at(2), wstride=8, t=_at(3), losses=_at(4), stats=_at(5), dl=_at(6),
             dx=_at(8), dw=_at(7), ws=_at(9), short=False)
    a.update(change)
    d = M.VocabularyDesc(a["dim"], a["vocab"], a["dtype"]) if a["desc"] else None
    need = L.mdlstm_vocabulary_workspace_bytes(d, a["rows"], backward)
    assert (need == 0) == (change in [c[0] for c in VOCABULARY_BAD])
    have = need - 1 if a["short"] else max(need, 1 << 16)
    head = (d, a["rows"], a["x"], a["xs"], a["w"], a["wstride"], a["t"])
    if backward:
        st = L.mdlstm_vocabulary_backward(*head, a["stats"], a["dl"], a["dx"], a["dw"], a["ws"], have, None)
    else:
        st = L.mdlstm_vocabulary_forward(*head, a["losses"], a["stats"], a["ws"], have, None)
    assert st == code, L.mdlstm_last_error()


def test_calls_of_nothing():
    M = _L()
    L = M.lib()
    r, g, v = M.RecurrenceDesc(4, 1, 0), M.GroupNormDesc(4, 2, 1, 0, 1e-5), M.VocabularyDesc(4, 9, 1)
    assert L.mdlstm_recurrence_forward(r, 0, 0, 0, None, None, None, 4, None, 4, None, None, None, None, FAKE, 256, None) == OK
    assert L.mdlstm_recurrence_backward(r, 0, 0, 0, None, None, None, 4, None, 4, None, None, None, 4, None, None, None, None, FAKE, 256,
                                        None) == OK
    assert L.mdlstm_recurrence_step(r, 0, None, 4, None, 4, None, 0, None, None, None) == OK
    assert L.mdlstm_group_norm_forward(g, 0, 0, 0, None, None, None, 4, None, None, None, None, None, FAKE, 256, None) == OK
    assert L.mdlstm_vocabulary_forward(v, 0, None, 4, FAKE, 4, None, None, None, _at(9), L.mdlstm_vocabulary_workspace_bytes(v, 0, 0),
                                       None) == OK


@pytest.mark.parametrize("rows", [0, 1, 63, 64, 65, 1000, 20000, 1 << 22])
@pytest.mark.parametrize("dim,vocab", [(1, 1), (64, 60), (1000, 130000), (65536, 70000), (20, 1 << 24)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_vocabulary_workspaces(rows, dim, vocab, dtype):
    """Every allowed size has a plan; it holds the operands' pieces at least, and a forward call's grows with the rows."""
    M = _L()
    d = M.VocabularyDesc(dim, vocab, dtype)
    fwd, bwd = (M.lib().mdlstm_vocabulary_workspace_bytes(d, rows, b) for b in (0, 1))
    assert 16 <= fwd < 1 << 44 and bwd < 1 << 44
    assert bwd >= rows * dim * 2 * (1 if dtype else 3) + rows * dim * 4


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    from paper_1902_11208_amd import sequence

    z, st = torch.zeros(5, 8), torch.zeros(9, 8)
    op = sequence.GatedRecurrence([2, 0, 3], 8, dtype=torch.float32, device="cpu")
    for a, b, state, says in ((z, z, None, "device"), (z[:4], z, None, "z has shape"), (z, z.double(), None, "x has dtype"),
                              (torch.zeros(5, 16)[:, ::2], z, None, "z must be contiguous"), (z, z, torch.zeros(3, 7), "state has shape"),
                              (torch.zeros(1, 8).expand(5, 8), z, None, "overlap"), (z, z, torch.zeros(8, 3).t(), "state must be contiguous"),
                              (torch.zeros(5, 20)[:, :8], z, None, "device")):
        with pytest.raises(ValueError, match=says):
            op.forward(a, b, state=state)
    with pytest.raises(ValueError, match="forward call"):
        op.backward(z)
    for bad in (dict(lengths=[1, -1]), dict(gate="tanh"), dict(channels=0), dict(channels=-3)):
        with pytest.raises(ValueError):
            sequence.GatedRecurrence(**{**dict(lengths=[3], channels=8, device="cpu"), **bad})
    with pytest.raises(TypeError):
        sequence.GatedRecurrence([3], 8, dtype=torch.float16, device="cpu")
    for change, says in ((dict(), "device"), (dict(z=torch.zeros(5, 8, 1)), "2 dimensions"), (dict(x=z[:3]), "x has shape"),
                         (dict(state=st.bfloat16()), "state has dtype"), (dict(state=torch.zeros(8, 9).t()), "state must be contiguous"),
                         (dict(slots=torch.zeros(5, dtype=torch.int64)), "slots has dtype"), (dict(out=torch.zeros(5, 16)[:, ::2]), "contiguous"),
                         (dict(gate="relu"), "gate")):
        with pytest.raises(ValueError, match=says):
            sequence.gated_recurrence_step(**{**dict(z=z, x=z, state=st), **change})
    with pytest.raises(TypeError):
        sequence.gated_recurrence_step(z.half(), z.half(), st)
    one = torch.ones(8)
    for bad in (dict(weight=torch.ones(2, 4)), dict(weight=one), dict(activation="gelu"), dict(weight=None), dict(lengths=[-1])):
        with pytest.raises(ValueError):
            sequence.GroupNorm(**{**dict(lengths=[3], weight=one, bias=one, groups=2), **bad})
    for bad in (torch.ones(8), torch.ones(4, 8), None):
        with pytest.raises(ValueError):
            sequence.VocabularyLoss(bad, 3)
    with pytest.raises(TypeError):
        sequence.VocabularyLoss(torch.ones(4, 8, dtype=torch.float16), 3)
