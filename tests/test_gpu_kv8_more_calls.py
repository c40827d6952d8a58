"""Calls on the 8-bit cache that lie between the usual ones: a token of many query heads on one, batches of long slices by the copy, moves between caches of
different layouts."""
import math

import numpy as np
import pytest

import block_util as bu
import kv8_util as ku
from gpu_util import dev_bf16, host_f64, say
from synth_inputs import bf16_bits_to_f64, normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def turned(cache):
    """The same cache with heads ahead of rows in memory."""
    return cache._replace(k_codes=cache.k_codes.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3),
                          v_codes=cache.v_codes.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))


@pytest.mark.parametrize("B,s,off,Hq,Hkv,D", [(2, 1, 700, 48, 1, 128), (1, 1, 0, 40, 1, 64), (1, 1, 5000, 140, 1, 64), (3, 2, 300, 66, 2, 128)])
def test_tokens_of_many_heads_on_one(sp, B, s, off, Hq, Hkv, D):
    """More rows of a kv head than the kernel of few takes, of one or two rows a head: attention and sums of weights."""
    say("kv8, tokens of %r" % ((B, s, off, Hq, Hkv, D),))
    L, N = 32, off + s
    bits = [normal_bf16((B, n, H, D), 81, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv))]
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(dev_bf16(bits[1]), dev_bf16(bits[2]), cache, 0)
    k, v = (ku.Cache(B, Hkv, D, L).append(bf16_bits_to_f64(b)).values for b in bits[1:])
    see = np.broadcast_to(np.arange(N) <= (off + np.arange(s))[:, None], (B, Hq, s, N))
    q = dev_bf16(bits[0])
    r = bu.Reference(bf16_bits_to_f64(bits[0]), k, v, see, 1 / math.sqrt(D))
    out, lse = sp.slimpipe_attn_fwd_kv8(q, turned(cache), off, 0, N)
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)
    got = host_f64(sp.slimpipe_attn_kv8_weights(q, turned(cache), lse, off, 0, N))
    want = r.p.reshape(B, Hkv, -1, N).sum(2)
    # each term off by the score's error and the lse's, both in r.f32 (the lse twice that), the sums by a step a term
    rel = 3.0 * r.f32.max() + 2.0 ** -20 + s * Hq // Hkv * 2.0 ** -24
    assert (np.abs(got - want) <= 1.01 * rel * want + 1e-30).all()


@pytest.mark.parametrize("B,s,off,Hq,Hkv,D,causal,begin", [(2, 600, 100, 8, 2, 64, True, 0), (3, 300, 700, 8, 1, 128, True, 260), (2, 550, 200, 8, 2, 128, False, 33)])
def test_batches_of_long_slices_by_the_copy(sp, B, s, off, Hq, Hkv, D, causal, begin):
    import torch
    say("kv8, copy %r" % ((B, s, off, Hq, Hkv, D, causal, begin),))
    L, N = 64, off + s
    bits = [normal_bf16((B, n, H, D), 82, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv))]
    cache = sp.KvCache8.empty(B, N + 40, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(dev_bf16(bits[1]), dev_bf16(bits[2]), cache, 0)
    cache.k_codes[:, N:] = 0x7f
    k, v = (ku.Cache(B, Hkv, D, L).append(bf16_bits_to_f64(b)).values for b in bits[1:])
    key = np.arange(N)
    see = np.broadcast_to((key >= begin) & ((key <= (off + np.arange(s))[:, None]) | (not causal)), (B, Hq, s, N))
    q = dev_bf16(bits[0])
    need = sp.slimpipe_attn_kv8_workspace_bytes(q, cache, off, begin, N, causal)
    assert sp.slimpipe_attn_kv8_call_path(sp.make_params(q, cache.k_codes, q, off, begin, N, causal, None), L, need).copy == 1
    whole = torch.full((need + 4096,), 0x5a, device="cuda", dtype=torch.uint8)
    for dtype in (sp.BF16, sp.F32):
        r = bu.Reference(bf16_bits_to_f64(bits[0]), k, v, see, 1 / math.sqrt(D), dtype == sp.BF16)
        out, lse = sp.slimpipe_attn_fwd_kv8(q, turned(cache), off, begin, N, causal, out_dtype=dtype, workspace=whole[:need])
        bu.check("out", host_f64(out), r.out, r.out_tol)
        bu.check("lse", host_f64(lse), r.lse, r.lse_tol)
    assert (whole[need:] == 0x5a).all()


@pytest.mark.parametrize("D,L", [(64, 16), (128, 64)])
def test_moves_between_layouts(sp, D, L):
    """From and to caches with heads ahead of rows, and of more heads side by side: the codes and scales of the plain move, nothing beside them."""
    import torch
    B, N, H, keep = 2, 300, 3, 133
    rows = [dev_bf16(normal_bf16((B, N, H, D), 83, t)) for t in "kv"]
    cache = sp.KvCache8.empty(B, N, H, D, L)
    sp.slimpipe_attn_kv8_store(*rows, cache, 0)
    index = torch.from_numpy(np.sort(np.random.RandomState(5).rand(B, H, N).argsort(-1)[..., :keep], -1).astype(np.int32)).cuda()
    want = sp.slimpipe_attn_kv8_gather(cache, index, sp.KvCache8.empty(B, keep, H, D, L))
    wide = [torch.full((B, keep + 9, 2 * H, D), 0x33, device="cuda", dtype=torch.uint8) for _ in range(2)]
    scales = [torch.full((B, -(-(keep + 9) // L), H), 0x33, device="cuda", dtype=torch.uint8) for _ in range(2)]
    to = sp.KvCache8(wide[0][:, :, H:], scales[0], wide[1][:, :, H:], scales[1], L)
    sp.slimpipe_attn_kv8_gather(turned(cache), index, to)
    blocks = -(-keep // L)
    for x, y in ((to.k_codes, want.k_codes), (to.v_codes, want.v_codes)):
        assert torch.equal(x[:, :keep], y) and (x[:, keep:] == 0x33).all()
    for x, y in ((to.k_scales, want.k_scales), (to.v_scales, want.v_scales)):
        assert torch.equal(x[:, :blocks], y) and (x[:, blocks:] == 0x33).all()
    assert all((x[:, :, :H] == 0x33).all() for x in wide)
    back = turned(sp.KvCache8.empty(B, keep, H, D, L))
    sp.slimpipe_attn_kv8_gather(cache, index, back)
    assert torch.equal(back.k_codes, want.k_codes) and torch.equal(back.v_codes, want.v_codes) and torch.equal(back.k_scales, want.k_scales)
