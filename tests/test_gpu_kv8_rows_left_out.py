"""Sums of attention weights over rows that have lse -infinity: such a row adds nothing, whatever its queries hold and whatever is in the keys that it alone
sees."""
import math

import pytest

from gpu_util import dev_bf16, say
from synth_inputs import normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


# rows, offset, heads, kv heads, head_dim, causal, rows without weight
SHAPES = [
    (1, 200, 8, 2, 128, True, [0]),
    (3, 200, 4, 1, 64, True, [1]),
    (3, 5000, 4, 4, 128, False, [0, 2]),                # the last one: rows of a wave behind it read it once more
    (8, 300, 4, 1, 128, True, [6, 7]),                  # 32 rows of a kv head, the most of a token call
    (90, 200, 4, 2, 128, True, [0, 33, 89]),
    (90, 700, 4, 4, 64, False, [5, 88, 89]),
    (300, 2000, 4, 1, 128, True, list(range(200, 300))),   # tiles that see every key of a workgroup, whole ones without a weight
    (300, 2000, 3, 1, 64, False, [0, 299]),
    (700, 0, 2, 2, 128, True, [0, 1, 640]),
]


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("s,off,Hq,Hkv,D,causal,left_out", SHAPES)
def test_rows_without_weight_that_are_not_finite(sp, s, off, Hq, Hkv, D, causal, left_out, value):
    """The bits of the call whose left-out rows are zeros; and the others' weights, each row's 1 in all."""
    import torch
    say("kv8 weights, rows left out %r" % ((s, off, Hq, Hkv, D, causal, left_out, value),))
    B, L, N = 2, 32, off + s
    k, v = (dev_bf16(normal_bf16((B, N, Hkv, D), 61, t)) for t in "kv")
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(k, v, cache, 0)
    q = dev_bf16(normal_bf16((B, s, Hq, D), 61, "q"))
    lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, 0, N, causal)[1]
    # (in the first sequence alone: those of the second keep their weight)
    lse[0, :, left_out] = -math.inf
    zero, bad = q.clone(), q.clone()
    zero[0, left_out] = 0.0
    bad[0, left_out] = value
    before = torch.rand((B, Hkv, N), device="cuda")
    for previous in (None, before):
        want = sp.slimpipe_attn_kv8_weights(zero, cache, lse, off, 0, N, causal, previous=previous, decay=0.5)
        got = sp.slimpipe_attn_kv8_weights(bad, cache, lse, off, 0, N, causal, previous=previous, decay=0.5)
        assert torch.equal(got, want)
    want = sp.slimpipe_attn_kv8_weights(zero, cache, lse, off, 0, N, causal)
    # (a row's terms are each off by less than 2^-11: D products of 2^-24 of their sizes, the lse, the exponential)
    for b, rows in ((0, s - len(left_out)), (1, s)):
        assert abs(float(want[b].double().sum()) - rows * Hq) <= rows * Hq * 2.0 ** -10


@pytest.mark.parametrize("s,off,Hq,Hkv,D", [(1, 40, 4, 1, 128), (4, 300, 8, 2, 64), (120, 300, 4, 1, 128), (300, 500, 2, 2, 64)])
def test_keys_that_only_rows_without_weight_see(sp, s, off, Hq, Hkv, D):
    """The last row is left out; its own key holds NaN codes: weight 0, and the others' weights as they are with numbers there."""
    import torch
    say("kv8 weights, key of a row left out %r" % ((s, off, Hq, Hkv, D),))
    B, L, N = 1, 16, off + s
    k, v = (dev_bf16(normal_bf16((B, N, Hkv, D), 62, t)) for t in "kv")
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(k, v, cache, 0)
    q = dev_bf16(normal_bf16((B, s, Hq, D), 62, "q"))
    lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, 0, N)[1]
    lse[..., -1] = -math.inf
    want = sp.slimpipe_attn_kv8_weights(q, cache, lse, off, 0, N)
    assert (want[..., -1] == 0).all()
    cache.k_codes[:, -1] = 0x7f
    assert torch.equal(sp.slimpipe_attn_kv8_weights(q, cache, lse, off, 0, N), want)
