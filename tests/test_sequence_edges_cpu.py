"""Host checks of the sequence operators at the edges of their range (runs
without a GPU: the addresses are never dereferenced)."""
import ctypes

import pytest

OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 4, 5


@pytest.fixture(scope="module", autouse=True)
def _built(built_lib):
    pass


def _L():
    from paper_1902_11208_amd import _lib

    return _lib


# --- outputs that overlap inputs or each other --------------------------------------------
N, TOKENS, LONGEST, HEADS, KV, DK, DV = 3, 100, 50, 4, 2, 32, 16
SIZES = dict(offsets=8 * (N + 1), order=4 * N, rates=4 * HEADS, q=TOKENS * 128 * 4, k=TOKENS * 64 * 4, v=TOKENS * 32 * 4,
             state=4 * N * HEADS * DK * DV, o=TOKENS * HEADS * DV * 4, final=4 * N * HEADS * DK * DV,
             grad_o=TOKENS * 64 * 4, dfinal=4 * N * HEADS * DK * DV, dq=TOKENS * HEADS * DK * 4, dk=TOKENS * KV * DK * 4,
             dv=TOKENS * KV * DV * 4, dstate=4 * N * HEADS * DK * DV)


def _apart():
    """Addresses of buffers that lie one after the other."""
    at, p = {}, 1 << 40
    for name, size in SIZES.items():
        at[name] = p
        p += size + 255 & ~255
    at["ws"] = p
    return at


def _need(backward):
    L = _L()
    return L.lib().mdlstm_attention_workspace_bytes(L.AttentionDesc(HEADS, KV, DK, DV, 0, 1.0), N, TOKENS, LONGEST, int(backward))


def _call(at, backward):
    import torch

    if torch.cuda.is_available():
        pytest.skip("the addresses are no memory of the device")
    L = _L()
    d = L.AttentionDesc(HEADS, KV, DK, DV, 0, 1.0)
    view = lambda n, ts, hs: L.Heads(at[n], ts, hs)  # noqa: E731
    need = _need(backward)
    qkv = view("q", 128, 32), view("k", 64, 32), view("v", 32, 16)
    tables = at["offsets"], at["order"], at["rates"]
    if backward:
        st = L.lib().mdlstm_attention_backward(d, N, TOKENS, LONGEST, *tables, *qkv, at["state"], view("grad_o", 64, 16),
                                               at["dfinal"], at["dq"], at["dk"], at["dv"], at["dstate"], at["ws"], need, None)
    else:
        st = L.lib().mdlstm_attention_forward(d, N, TOKENS, LONGEST, *tables, *qkv, at["state"], at["o"], at["final"],
                                              at["ws"], need, None)
    return st, L.lib().mdlstm_last_error().decode()


@pytest.mark.parametrize("out,other,backward", [
    ("final", "state", False), ("o", "q", False), ("o", "k", False), ("o", "v", False), ("final", "q", False),
    ("final", "o", False), ("o", "state", False), ("o", "offsets", False), ("final", "rates", False), ("ws", "q", False),
    ("ws", "final", False), ("dstate", "dfinal", True), ("dstate", "state", True), ("dq", "q", True), ("dk", "k", True),
    ("dv", "grad_o", True), ("dq", "dk", True), ("dk", "dv", True), ("dstate", "dq", True), ("dv", "order", True),
    ("ws", "dfinal", True)])
def test_attention_refuses_outputs_that_overlap(out, other, backward):
    """The same start, and an output whose first 256 bytes are the last of the other buffer or the other way round."""
    at = _apart()
    size = _need(backward) if out == "ws" else SIZES[out]
    for p in (at[other], at[other] + max(0, SIZES[other] - 256) // 256 * 256, at[other] - (size - 256) // 256 * 256):
        st, says = _call(dict(at, **{out: p}), backward)
        assert st == INVALID and "overlap" in says, (st, says)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_accepts_buffers_that_touch(backward):
    """Buffers one right after the other pass the checks (and the call then finds no device)."""
    st, says = _call(_apart(), backward)
    assert st not in (OK, INVALID, WORKSPACE, UNSUPPORTED) and "overlap" not in says, (st, says)


# --- where sequences are cut into segments: the workspace then holds states -----------------------------------
@pytest.mark.parametrize("n,tokens,heads,dim,dtype,forward,backward", [
    (1, 384, 4, 32, 0, False, False), (1, 512, 4, 32, 0, True, True), (1, 512, 8, 64, 1, True, True),
    (8, 512, 4, 32, 0, True, False), (16, 512, 4, 32, 0, False, False), (4, 1024, 8, 64, 1, True, True),
    (16, 1024, 8, 64, 1, False, False), (16, 2048, 8, 64, 1, True, False), (32, 2048, 8, 64, 1, False, False),
    (8, 2048, 4, 128, 1, True, False), (16, 2048, 4, 128, 1, True, False), (64, 2048, 4, 128, 1, False, False),
    (1, 65536, 8, 64, 1, True, True)])
def test_segments_only_where_they_are_faster(n, tokens, heads, dim, dtype, forward, backward):
    L = _L()
    d = L.AttentionDesc(heads, heads, dim, dim, dtype, 1.0)
    for b, want in ((0, forward), (1, backward)):
        size = L.lib().mdlstm_attention_workspace_bytes(d, n, n * tokens, tokens, b)
        assert (size > 256) == want, (b, size)
