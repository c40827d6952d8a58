"""Eviction again and again between two 8-bit caches and their sums, whose memory is used over: entries of rows that come later are set to 0 by the caller, as
the move leaves them."""
import math

import numpy as np
import pytest

from gpu_util import host_f64, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


@pytest.mark.parametrize("step", [3, 40])
def test_sums_over_several_evictions(sp, step):
    """Slices of tokens or of a few rows; the sums of every row that is there against 64 bits, from its first call on."""
    import torch
    say("kv8, evictions between two caches, %d rows a call" % step)
    B, Hq, Hkv, D, L, N, keep, recent, decay = 2, 8, 2, 64, 16, 240, 70, 9, 0.5
    g = torch.Generator(device="cuda").manual_seed(99)
    caches = [sp.KvCache8.empty(B, N, Hkv, D, L) for _ in range(2)]
    sums = [torch.full((B, Hkv, N), 7.0, device="cuda") for _ in range(2)]
    now, n, want, rel = 0, 0, np.zeros((B, Hkv, 0)), 0.0
    sums[0].zero_()
    for call in range(4 * (N - keep) // step):
        if n + step > N:
            order = np.argsort(-np.float64(sums[now].cpu().numpy()[..., :n - recent]), axis=-1, kind="stable")[..., :keep - recent]
            expect = np.concatenate([np.sort(order, -1), np.broadcast_to(np.arange(n - recent, n), (B, Hkv, recent))], -1)
            index = sp.slimpipe_attn_kv8_keep(sums[now], n, keep, recent)
            assert np.array_equal(index.cpu().numpy(), expect)
            other = 1 - now
            assert (sums[other][..., keep:] != 0).any()
            sp.slimpipe_attn_kv8_gather(caches[now], index, caches[other], sums[now], sums[other])
            sums[other][..., keep:] = 0
            now, n, want = other, keep, np.take_along_axis(want, expect, -1)
        q = torch.randn((B, step, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
        k, v = torch.randn((2, B, step, Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
        sp.slimpipe_attn_kv8_store(k, v, caches[now], n)
        _, lse = sp.slimpipe_attn_fwd_kv8(q, caches[now], n, 0, n + step)
        sp.slimpipe_attn_kv8_weights(q, caches[now], lse, n, 0, n + step, weights=sums[now], previous=sums[now], decay=decay)
        keys = np.repeat(host_f64(sp.slimpipe_attn_kv8_load(caches[now], 0, n + step)[0]).transpose(0, 2, 1, 3), Hq // Hkv, 1)
        x = host_f64(q).transpose(0, 2, 1, 3) @ keys.swapaxes(-1, -2) / math.sqrt(D)
        p = np.where(np.arange(n + step) <= n + np.arange(step)[:, None], np.exp(x - host_f64(lse)[..., None]), 0.0)
        n += step
        want = decay * np.pad(want, ((0, 0), (0, 0), (0, n - want.shape[-1]))) + p.reshape(B, Hkv, -1, n).sum(2)
        # a score, of D products, is off by D 2^-24 of their sizes, the exponential and the sums by 2^-20 and a step a term; earlier sums keep their relative error
        size = np.abs(host_f64(q)).max() * np.abs(keys).max() * math.sqrt(D)
        rel = max(rel, D * 2.0 ** -24 * size + 2.0 ** -20 + (step * Hq // Hkv + 4) * 2.0 ** -24)
        assert (np.abs(host_f64(sums[now])[..., :n] - want) <= (rel + call * 2.0 ** -23) * want + 1e-30).all(), call
