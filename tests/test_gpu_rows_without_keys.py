"""Rows that see no key have out 0, lse -infinity and no gradient, whatever the keys hold that other rows of the call see."""
import pytest

from gpu_util import dev_bf16, say
from synth_inputs import normal_bf16

pytestmark = pytest.mark.gpu

# rows, heads, kv heads; the range begins behind the first rows
SHAPES = [(3, 4, 1), (2, 4, 4), (20, 4, 1), (300, 4, 2), (1500, 8, 8)]
OFF = 640


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def case(s, Hq, Hkv, D, bad):
    N, begin = OFF + s, OFF + 1 + (s // 2 if s > 20 else 0)
    q, k, v, do = (dev_bf16(normal_bf16((1, n, h, D), 51, t)) for t, n, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv), ("do", s, Hq)))
    v[0, begin] = bad
    v[0, N - 1, :, ::3] = bad
    return q, k, v, do, N, begin, begin - OFF


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_cache_forward(sp, shape, D, bad):
    import torch
    say("kv4 rows without keys %r D=%d %r" % (shape, D, bad))
    q, k, v, _, N, begin, none = case(*shape, D, bad)
    cache = sp.KvCache4.empty(1, N, shape[2], D)
    sp.slimpipe_attn_kv4_store(k, v, cache, 0)
    for dtype in (sp.BF16, sp.F32):
        out, lse = sp.slimpipe_attn_fwd_kv4(q, cache, OFF, begin, N, out_dtype=dtype)
        assert (out[:, :none] == 0).all() and (lse[:, :, :none] == -float("inf")).all()
        assert torch.isnan(out[:, none:, :, 0]).all() and torch.isfinite(lse[:, :, none:]).all()      # the others do see it
