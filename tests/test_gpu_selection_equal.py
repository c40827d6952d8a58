"""Block selection where scores are equal or not finite: every row of the index is whole, ascending and the one that 64-bit scores give, with lists
of every length that the kernels have (top_k up to 8, 16, 32, 64), for few rows and for many."""
import numpy as np
import pytest

from gpu_util import dev_bf16, host_f64, say
from synth_inputs import normal_bf16

pytestmark = pytest.mark.gpu

HQ, L, NB = 8, 64, 150


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def whole(index, off, top_k, blocks):
    """Every row: min(top_k, blocks that it may have) entries, ascending, its own block the last of them, then -1."""
    B, H, s, _ = index.shape
    own = (off + np.arange(s)) // L
    n = np.minimum(top_k, own + 1)
    assert (own < blocks).all()
    slot = np.arange(top_k)
    filled = np.broadcast_to(slot < n[:, None], index.shape)
    assert (index[filled] >= 0).all() and (index[~filled] == -1).all()
    assert (np.diff(index, axis=-1)[np.broadcast_to(slot[1:] < n[:, None], (B, H, s, top_k - 1))] > 0).all()
    last = np.take_along_axis(index, np.broadcast_to((n - 1)[:, None], (B, H, s, 1)), -1)
    assert (last[..., 0] == own).all()


def first_blocks(s, off, top_k):
    """All scores equal: the lowest blocks and the row's own."""
    own = (off + np.arange(s)) // L
    n = np.minimum(top_k, own + 1)
    slot = np.arange(top_k)
    return np.where(slot < (n - 1)[:, None], slot, np.where(slot == (n - 1)[:, None], own[:, None], -1))


@pytest.mark.parametrize("top_k", [5, 8, 16, 24, 63, 64])
@pytest.mark.parametrize("s", [5, 4200])
def test_equal_scores(sp, s, top_k):
    """Rows of zeros on any means; any rows on means that are all zero, all one, all the same, or the same with a NaN row among them: the lowest indices,
    with more equal ones than a row's list has room for."""
    import torch
    D, off = 128, NB * L
    say("select equal s=%d top_k=%d" % (s, top_k))
    blocks = -(-(off + s) // L)
    base = dev_bf16(normal_bf16((1, blocks, 1, D), 41, "k"))[:, :, 0].float()[:, None]
    q = dev_bf16(normal_bf16((1, s, HQ, D), 41, "q"))
    zero = torch.zeros_like(q)
    zero[:, ::2] = -0.0
    same = base[:, :, :1].expand_as(base).contiguous()
    want = first_blocks(s, off, top_k)
    cases = [(zero, base), (q, torch.zeros_like(base)), (q, torch.full_like(base, -0.0)), (q, torch.ones_like(base)), (q, same), (q * 2.0 ** -60, same), (q, same * 2.0 ** -120)]
    for x, m in cases:
        got = sp.slimpipe_attn_block_select(x, m.contiguous(), off, 0, off + s, L, top_k).cpu().numpy()
        whole(got, off, top_k, blocks)
        assert (got == want).all()
    # a block of NaN among equal ones is passed over
    m = same.clone()
    m[0, 0, 2] = float("nan")
    got = sp.slimpipe_attn_block_select(q, m, off, 0, off + s, L, top_k).cpu().numpy()
    whole(got, off, top_k, blocks)
    want = want.copy()
    want[:, :top_k - 1] += want[:, :top_k - 1] >= 2           # (there are more than top_k before every row's own)
    assert (got == want).all()


@pytest.mark.parametrize("top_k", [5, 12, 24, 63, 64])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("s", [5, 4200])
def test_two_levels(sp, s, D, top_k):
    """Equal scores on both sides of the last place: means of ones, some of them larger by what 32 bits do not show."""
    import torch
    off = NB * L
    say("select two levels s=%d D=%d top_k=%d" % (s, D, top_k))
    blocks = -(-(off + s) // L)
    q = torch.ones((1, s, HQ, D), device="cuda", dtype=torch.bfloat16)
    q[:, 1::2] = 2.0
    up = np.sort(np.random.default_rng(top_k).permutation(NB)[:top_k // 2])
    m = torch.zeros((1, 1, blocks, D), device="cuda")
    m[..., 0] = 1.0
    m[0, 0, up, 1] = 2.0 ** -40
    got = sp.slimpipe_attn_block_select(q, m, off, 0, off + s, L, top_k).cpu().numpy()
    whole(got, off, top_k, blocks)
    rest = np.setdiff1d(np.arange(NB), up)[:top_k - 1 - len(up)]
    assert (got[..., :top_k - 1] == np.sort(np.concatenate([up, rest]))).all()


@pytest.mark.parametrize("top_k", [5, 16, 24, 64])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("s", [5, 4200])
def test_rows_are_whole_whatever_the_scores(sp, s, D, top_k):
    """Zeros, tiny, huge, infinite and NaN rows on ordinary, tiny, nearly equal, half zero and not finite means: entries, order, own block and fill-up; and no
    block that is left out has a score above one that is taken, of equal ones no lower index.  Scores are float64 sums in numpy's order: one that is off
    by D 2^-53 of its terms on either side may go either way."""
    import torch
    off = 20 * L                                              # few blocks before the first rows: -1 behind them
    say("select whole rows s=%d D=%d top_k=%d" % (s, D, top_k))
    blocks = -(-(off + s) // L)
    q = dev_bf16(normal_bf16((1, s, HQ, D), 42, "q"))
    q[:, torch.arange(s, device="cuda") % 5 == 1] = 0.0
    q[:, torch.arange(s, device="cuda") % 5 == 2] *= 2.0 ** -60
    q[0, 4::50, 1] *= 2.0 ** 100
    q[0, 4::50, 2, 3] = float("inf")
    q[0, 4::50, 3, 3] = float("nan")
    base = dev_bf16(normal_bf16((1, blocks, 1, D), 42, "k"))[:, :, 0].float()[:, None].contiguous()
    half, bad = base.clone(), base.clone()
    half[:, :, ::2] = 0.0
    for j, d, v in ((7, 1, float("nan")), (9, 2, float("inf")), (11, 2, -float("inf"))):
        bad[0, 0, j, d] = v
    q64 = host_f64(q)[0]
    own = (off + np.arange(s)) // L
    j = np.arange(blocks)
    for m in (base, base * 2.0 ** -60, base * 2.0 ** -110, 1.0 + base * 2.0 ** -22, half, bad):
        got = sp.slimpipe_attn_block_select(q, m, off, 0, off + s, L, top_k).cpu().numpy()
        whole(got, off, top_k, blocks)
        m64 = host_f64(m)[0, 0]
        for h in range(HQ):
            with np.errstate(invalid="ignore", over="ignore"):
                x = q64[:, h] @ m64.T
                slack = D * 2.0 ** -53 * (np.abs(q64[:, h]) @ np.abs(m64).T)
            # as numbers in order: NaN below -infinity below all others
            key = np.where(np.isnan(x), -np.inf, np.maximum(x, -1e308))
            slack = np.where(np.isfinite(slack), slack, 0.0)
            taken = np.zeros((s, blocks), dtype=bool)
            np.put_along_axis(taken, np.where(got[0, h] < 0, own[:, None], got[0, h]), True, -1)
            free = j < own[:, None]
            kept, left = taken & free, ~taken & free
            # the lowest kept and the highest that was left, as far as rounding can tell; equal ones by index
            low = np.where(kept, key + slack, np.inf).min(-1)
            high = np.where(left, key - slack, -np.inf).max(-1, initial=-np.inf)
            assert (high <= low).all(), h
            exact = ~np.any(slack > 0, -1)                     # rows of zeros: no rounding at all
            for r in np.nonzero(exact & left.any(-1) & kept.any(-1))[0]:
                worst = key[r][kept[r]].min()
                assert not (key[r][left[r]] > worst).any()
                at = j[kept[r] & (key[r] == worst)].max()
                assert (j[left[r] & (key[r] == worst)] > at).all(), (h, r)
