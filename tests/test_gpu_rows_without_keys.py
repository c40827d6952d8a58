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


def all_blocks(N, L, s, Hq):
    """Every row names the last 40 blocks."""
    import torch
    blocks = -(-N // L)
    return torch.arange(max(0, blocks - 40), blocks, device="cuda", dtype=torch.int32).expand(1, Hq, s, min(40, blocks)).contiguous()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_sparse_forward_and_backward(sp, shape, D, bad):
    import torch
    s, Hq, Hkv = shape
    say("sparse rows without keys %r D=%d %r" % (shape, D, bad))
    q, k, v, do, N, begin, none = case(*shape, D, bad)
    k[0, begin + 1:begin + 2] = torch.where(torch.arange(D, device="cuda") == 5, float("nan"), 0.0).to(torch.bfloat16)
    index = all_blocks(N, 64, s, Hq)
    for dtype in (sp.BF16, sp.F32):
        out, lse = sp.slimpipe_attn_block_fwd(q, k, v, index, OFF, begin, N, 64, out_dtype=dtype)
        assert (out[:, :none] == 0).all() and (lse[:, :, :none] == -float("inf")).all()
        assert not torch.isfinite(out[:, none:, :, 0]).any()
        dk, dv = torch.zeros((2,) + k.shape, device="cuda")
        dq = sp.slimpipe_attn_block_bwd(q, k, v, index, out.bfloat16(), do, lse, OFF, begin, N, 64, dk, dv, dq_dtype=dtype)
        assert (dq[:, :none] == 0).all()
        assert (dk[:, :begin] == 0).all() and (dv[:, :begin] == 0).all()
    dq = torch.full((1, s, Hq, D), 3.0, device="cuda")
    sp.slimpipe_attn_block_bwd(q, k, v, index, out.bfloat16(), do, lse, OFF, begin, N, 64, dk, dv, dq=dq, dq_dtype=sp.F32, dq_accumulate=True)
    assert (dq[:, :none] == 3.0).all()
