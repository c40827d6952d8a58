"""Long slices on the 8-bit cache in less workspace than they ask for: every way that a call then goes, against 64 bits, nothing written beyond the room."""
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


# batch, rows, heads, kv heads, head_dim, offset, kv_begin, room in ranges (beside a copy or alone), what the call takes
CASES = [
    (1, 257, 8, 1, 128, 3000, 0, False, 0, (0, 1, 128)),
    (1, 257, 8, 1, 128, 3000, 0, False, 2, (0, 2, 128)),
    (1, 257, 8, 1, 128, 3000, 0, False, 3, (0, 3, 128)),
    (1, 257, 8, 1, 128, 3000, 0, False, 5, (1, 3, 0)),       # what the dense call asks for fits beside the copy
    (1, 1030, 4, 2, 64, 6000, 0, True, 0, (0, 3, 128)),
    (1, 1030, 4, 2, 64, 6000, 2000, True, 0, (1, 1, 0)),     # fewer keys: the dense call asks for no range
    (1, 2100, 8, 8, 128, 300, 0, False, 2, (0, 2, 256)),     # 72 blocks of 256 rows: eight waves from two ranges on
    (1, 2100, 8, 8, 128, 300, 0, True, 0, (1, 1, 0)),        # no second range fits: the copy undivided
    (1, 2048, 1, 1, 64, 100, 0, False, 0, (0, 1, 128)),
]


@pytest.mark.parametrize("B,s,Hq,Hkv,D,off,begin,copy,ranges,takes", CASES)
def test_forward_in_little_room(sp, B, s, Hq, Hkv, D, off, begin, copy, ranges, takes):
    import torch
    say("kv8 forward in little room %r" % ((B, s, Hq, Hkv, D, off, begin, copy, ranges),))
    L, N = 64, off + s
    bits = [normal_bf16((B, n, H, D), 71, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv))]
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(dev_bf16(bits[1]), dev_bf16(bits[2]), cache, 0)
    k, v = (ku.Cache(B, Hkv, D, L).append(bf16_bits_to_f64(b)).values for b in bits[1:])
    q = dev_bf16(bits[0])
    room = (4 * D * B * Hkv * (N - begin) + 512 if copy else 0) + (ranges * B * Hq * s * (D + 1) * 4 + 1024 if ranges else 0)
    p = sp.make_params(q, cache.k_codes, q, off, begin, N, True, None)
    path = sp.slimpipe_attn_kv8_call_path(p, L, room)
    assert (path.copy, path.ranges, path.workgroup_rows) == takes
    whole = torch.full((room + 4096,), 0x5a, device="cuda", dtype=torch.uint8)
    key = np.arange(N)
    see = np.broadcast_to((key >= begin) & (key <= (off + np.arange(s))[:, None]), (B, Hq, s, N))
    r = bu.Reference(bf16_bits_to_f64(bits[0]), k, v, see, 1 / math.sqrt(D))
    out, lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, begin, N, workspace=whole[:room])
    assert (whole[room:] == 0x5a).all()
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)
    again = sp.slimpipe_attn_fwd_kv8(q, cache, off, begin, N, workspace=whole[:room])
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
