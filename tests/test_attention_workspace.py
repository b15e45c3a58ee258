"""The workspace of attention's gradients (CPU): the room for the sinks' shares goes by the
rows, not by the samples."""
from __future__ import annotations

import os

import pytest


@pytest.fixture(scope="module")
def need():
    from paper_1505_02890_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_1505_02890_amd.build import build
        build()
    return _lib.lib().scn_attn_bwd_workspace_bytes


@pytest.mark.parametrize("n", [1, 255, 257, 100_000, 200_001, 10_000_000])
@pytest.mark.parametrize("H,K,D", [(8, 8, 128), (4, 1, 64), (3, 3, 24)])
@pytest.mark.parametrize("left", [0, 30, 1000])
@pytest.mark.parametrize("sinks", [1, 63, 256])
def test_shares_go_by_the_rows(need, n, H, K, D, left, sinks):
    rows = need(n, 1, D, H, K, -1, 0)  # what a row takes without shares
    assert 4 * n * H <= rows <= 16 * (n * H + 64)
    most = (n // 256 + 1) + n // (left + 256)  # shares of 256 queries or more
    for batch in (1, 32, 5000, 1_000_000):
        shares = need(n, batch, D, H, K, left, sinks) - rows
        assert 0 <= shares <= most * K * min(sinks, n) * 2 * D * 4
    # at most twice the keys and values in fp32, for 256 sinks
    assert need(n, n, D, H, K, left, 256) - rows <= 2 * (2 * n * K * D * 4) + K * 256 * 2 * D * 4
