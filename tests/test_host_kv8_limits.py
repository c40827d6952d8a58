"""CPU-only checks of the largest calls on the 8-bit cache: what the header states as a limit is what is refused, with which code."""
import ctypes

import pytest

SHAPE = -2
A, WS = 0x1000, 1 << 50            # an address that is never read: a call is refused first


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def params(sp, s_q, batch, heads, keys, offset):
    D = 64
    row = heads * D
    return sp.AttnParams(batch, s_q, heads, heads, D, 1, keys, offset, 0, keys, 0.125, sp.BF16, s_q * row, row, D, keys * row, row, D, s_q * row, row, D)


@pytest.mark.parametrize("s_q", [1, 33, 500])
def test_sums_of_weights_count_less_than_2_32_threads(sp, s_q):
    """A workgroup of 256 threads for every 256 keys of a plane, rounded up to eights."""
    for batch, heads, keys, code in ((2, 4, ((1 << 21) - 1) * 256, 0), (2, 4, ((1 << 21) - 1) * 256 + 1, SHAPE), (1, 4, 1 << 30, SHAPE), (1, 2, 1 << 30, 0),
                                     (4, 16, ((1 << 18) - 1) * 256 + 1, SHAPE), (4, 16, 1 << 25, 0), (4, 8, 1 << 28, SHAPE)):
        p, n = params(sp, s_q, batch, heads, keys, keys - s_q), ctypes.c_size_t(0)
        assert sp.lib.slimpipe_attn_kv8_weights_workspace_bytes(ctypes.byref(p), 64, ctypes.byref(n)) == code, (batch, heads, keys)
        if code:
            assert sp.lib.slimpipe_attn_kv8_weights(ctypes.byref(p), 64, A, A, A, A, None, 1.0, A, A, WS, None) == code
