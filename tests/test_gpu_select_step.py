"""A step of the selection as a decoder or trainer takes it: the slice's means into a buffer that holds nothing valid there yet, then the choice."""
import numpy as np
import pytest

import block_util as bu
from gpu_util import dev_bf16, host_f64, say
from synth_inputs import bf16_bits_to_f64, normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


# batch, rows, offset, heads, kv heads, head_dim, block, top_k
@pytest.mark.parametrize("case", [(1, 1, 700, 8, 1, 128, 64, 5), (4, 1, 1023, 8, 1, 128, 256, 3), (2, 130, 511, 4, 2, 64, 64, 4), (1, 257, 0, 2, 2, 128, 192, 2),
                                  (3, 100, 901, 6, 3, 64, 128, 24), (1, 4200, 333, 8, 1, 128, 64, 8)])
def test_means_of_the_slice_are_made_by_the_call(sp, case):
    """All blocks from the slice's first on hold NaN before: the call makes every one of them, to the last partial block, and nothing else."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = case
    say("select step %r" % (case,))
    N, first = off + s, off // L
    bits = {t: normal_bf16((B, n, H, D), 44, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv))}
    q, k, k64 = dev_bf16(bits["q"]), dev_bf16(bits["k"]), bf16_bits_to_f64(bits["k"])
    blocks = -(-N // L)
    means = torch.full((B, Hkv, blocks + 1, D), float("nan"), device="cuda")
    exact = bu.means(k64, 0, N, L)
    for j in range(first):
        means[:, :, j] = torch.from_numpy(exact[j].astype(np.float32)).cuda()
    sp.slimpipe_attn_block_means(torch.nn.functional.pad(k, (0, 0, 0, 0, 0, (blocks + 1) * L - N)), first * L, N, L, means=means)
    got = host_f64(means)
    for j in range(blocks):
        # a mean in 64 bits, one rounding to 32
        assert (np.abs(got[:, :, j] - exact[j]) <= 2.0 ** -24 * np.abs(exact[j]) + 2.0 ** -50 * np.abs(k64).max()).all(), j
    assert np.isnan(got[:, :, blocks]).all()                  # behind the slice: untouched
    index = sp.slimpipe_attn_block_select(q, means[:, :, :blocks].contiguous(), off, 0, N, L, top_k).cpu().numpy()
    if s < 1000:
        assert np.array_equal(index, bu.select(bf16_bits_to_f64(bits["q"]), got[:, :, :blocks], off, 0, N, L, top_k, True))
    own = (off + np.arange(s)) // L
    assert (index.max(-1) == own).all()
