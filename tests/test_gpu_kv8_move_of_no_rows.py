"""A move to another 8-bit cache where whole blocks have no row: rows of zeros with the format's least scale, behind which rows are appended as usual."""
import numpy as np
import pytest

import kv8_util as ku
from gpu_util import dev_bf16, host_f64, say
from synth_inputs import normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


@pytest.mark.parametrize("H,D,L", [(1, 64, 16), (3, 128, 32), (2, 64, 256)])
def test_blocks_of_entries_that_are_no_row(sp, H, D, L):
    import torch
    say("kv8 gather, blocks without a row %r" % ((H, D, L),))
    N, keep = 2 * L + 5, 3 * L + 3
    rows = [dev_bf16(normal_bf16((1, N, H, D), 63, t)) for t in "kv"]
    cache = sp.KvCache8.empty(1, N, H, D, L)
    sp.slimpipe_attn_kv8_store(*rows, cache, 0)
    # the first block has every second row, the second and the last none, the third one row, in the last head alone
    index = torch.full((1, H, keep), -1, device="cuda", dtype=torch.int32)
    index[..., 0:L:2] = torch.arange(0, L, 2, device="cuda", dtype=torch.int32)
    index[..., L:2 * L] = N
    index[:, -1, 2 * L + 1] = N - 1
    kept = sp.KvCache8(*(x.fill_(0x55) for x in sp.KvCache8.empty(1, keep + L, H, D, L)[:4]), L)
    sp.slimpipe_attn_kv8_gather(cache, index, kept)
    at = index[0].cpu().numpy()
    there = (at >= 0) & (at < N)
    for x, y, scales in zip(rows, sp.slimpipe_attn_kv8_load(kept, 0, keep), (kept.k_scales, kept.v_scales)):
        from_ = ku.Cache(1, H, D, L).append(host_f64(x))
        byte = np.full((4, H), ku.LEAST + 127)
        for h in range(H):
            for j in range(4):
                r = at[h, j * L:(j + 1) * L]
                byte[j, h] = max([ku.LEAST + 127] + [int(from_.scales()[0, i // L, h]) for i in r if 0 <= i < N])
        assert np.array_equal(scales[0, :4].cpu().numpy(), byte)
        values = np.where(there[..., None], from_.values[0].swapaxes(0, 1)[np.arange(H)[:, None], np.where(there, at, 0)], 0.0)
        want = ku.round_to(values, np.repeat(2.0 ** (byte - 127.0), L, 0)[:keep].T[..., None])
        assert np.array_equal(host_f64(y)[0].swapaxes(0, 1), want)
    # a row behind them: the block's rows are zeros still, its scale is the row's
    more = [x[:, :1].clone() for x in rows]
    sp.slimpipe_attn_kv8_store(*more, kept, keep)
    for x, y, scales in zip(more, sp.slimpipe_attn_kv8_load(kept, 3 * L, keep + 1), (kept.k_scales, kept.v_scales)):
        alone = ku.Cache(1, H, D, L).append(host_f64(x))
        assert (y[:, :-1] == 0).all() and np.array_equal(host_f64(y)[:, -1:], alone.values)
        assert np.array_equal(scales[0, 3].cpu().numpy(), alone.scales()[0, 0])
