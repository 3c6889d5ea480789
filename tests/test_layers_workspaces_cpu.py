"""Workspaces of the group norm and the recurrence for thousands of short sequences with a long one among them, which is
taken in segments: what the short ones need on top stays below what their inputs hold. Host code only."""
import pytest


@pytest.fixture(scope="module", autouse=True)
def _built(built_lib):
    pass


BATCHES = [(1 << 20, 1, 3000), (70000, 1, 9000), (70000, 1, 300000), (5000, 40, 50000)]  # short ones, their tokens, the long one's


@pytest.mark.parametrize("n,short,long", BATCHES)
@pytest.mark.parametrize("channels,groups,dtype", [(512, 32, 1), (64, 4, 0), (2048, 32, 1)])
def test_group_norm(n, short, long, channels, groups, dtype):
    from paper_1902_11208_amd import _lib

    d = _lib.GroupNormDesc(channels, groups, dtype, 2, 1e-5)
    tokens = n * short + long
    for backward in (0, 1):
        need = _lib.lib().mdlstm_group_norm_workspace_bytes(d, n + 1, tokens, long, backward)
        # two numbers for each group of every sequence (forward: and of segments), and once more the same; 4096 shares of dw and db at most
        assert 16 <= need <= 2 * (n + 1 + tokens // 64) * groups * 8 + 4096 * 8 * max(channels, 512) + 4096, need


@pytest.mark.parametrize("n,short,long", BATCHES)
@pytest.mark.parametrize("channels,dtype", [(512, 1), (64, 0), (2048, 1)])
def test_recurrence(n, short, long, channels, dtype):
    from paper_1902_11208_amd import _lib

    tokens = n * short + long
    for backward in (0, 1):
        need = _lib.lib().mdlstm_recurrence_workspace_bytes(_lib.RecurrenceDesc(channels, dtype, 1), n + 1, tokens, long, backward)
        # three numbers for each edge between segments of 256 tokens at least
        assert 16 <= need <= 3 * (tokens // 256 + 1) * channels * 4 + 16, need
