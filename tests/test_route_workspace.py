"""The router's statistics workspace, without a GPU: one sized for the largest
batch does for every smaller one, and no tokens need hardly any."""
import numpy as np
import pytest

import paper_2606_04101_amd as uep

SIZES = sorted({0, 1, 15, 16, 17, 31, 33, 255, 4096, 8191, 8192, 8193, 16383, 16384, 16385, 32768, 32769, 65536, 1 << 20,
                (1 << 23) - 1, 1 << 23, *np.random.default_rng(1).integers(1, 1 << 23, 150).tolist(),
                *np.random.default_rng(2).integers(1, 40000, 300).tolist()})


@pytest.mark.parametrize("E", [1, 64, 65, 256, 1024])
@pytest.mark.parametrize("seq_len", [0, 1, 16, 17, 33, 700, 1024, 5000, 16384, 1 << 20, 1 << 40])
def test_workspace_does_not_shrink_with_more_tokens(E, seq_len):
    r = uep.Router(E, 1, seq_len=seq_len)
    got = [uep.ultraep_route_ws_bytes(T, r) for T in SIZES]
    for a, b, T in zip(got, got[1:], SIZES[1:]):
        assert a <= b, T
    # partials of 2 E + 1 words, of about as many workgroups as run at once
    assert got[-1] <= (2 * 1024 + 2) * (2 * E + 1) * 4


@pytest.mark.parametrize("seq_len", [0, 1, 1 << 20, (1 << 63) - 1])
def test_no_tokens_need_no_partials(seq_len):
    assert uep.ultraep_route_ws_bytes(0, uep.Router(256, 8, seq_len=seq_len)) <= 64
