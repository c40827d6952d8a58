"""The selection's order among scores that are no ordinary numbers."""
import numpy as np
import pytest

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


@pytest.mark.parametrize("nb,top_k", [(8, 5), (8, 7), (150, 5), (150, 12), (150, 24), (150, 64)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("s", [5, 4200])
def test_nan_comes_behind_minus_infinity(sp, s, D, nb, top_k):
    """More blocks with a score of -infinity or NaN than places: the infinite ones first, whatever their indices."""
    import torch
    Hq, L = 8, 64
    say("select NaN s=%d D=%d blocks=%d top_k=%d" % (s, D, nb, top_k))
    q = torch.ones((1, s, Hq, D), device="cuda", dtype=torch.bfloat16)
    means = torch.full((1, 1, nb, D), float("nan"), device="cuda")
    scores = np.full(nb, np.nan)
    for j, v in ((1, 1.0), (4, 2.0), (5, -np.inf), (nb - 1, -np.inf), (nb - 2, -3.0)):
        means[0, 0, j] = 0.0
        means[0, 0, j, 3] = v
        scores[j] = v
    order = sorted(range(nb), key=lambda j: (np.isnan(scores[j]), -scores[j] if scores[j] == scores[j] else 0.0, j))
    want = torch.tensor(sorted(order[:top_k]), device="cuda", dtype=torch.int32)
    got = sp.slimpipe_attn_block_select(q, means, 0, 0, nb * L, L, top_k, causal=False)
    assert torch.equal(got, want.expand(1, Hq, s, top_k)), got[0, 0, 0]
    # the same as the blocks before the rows' own, which takes a place
    more = -(-s // L)
    means = torch.cat([means, torch.zeros((1, 1, more, D), device="cuda")], 2)
    got = sp.slimpipe_attn_block_select(q, means, nb * L, 0, nb * L + s, L, top_k)
    want = torch.tensor(sorted(order[:top_k - 1]) + [nb], device="cuda", dtype=torch.int32)
    rows = min(s, L)                                          # (behind them the blocks of zeros compete)
    assert torch.equal(got[:, :, :rows], want.expand(1, Hq, rows, top_k)), got[0, 0, 0]
