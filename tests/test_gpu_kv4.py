"""The key/value cache in 4 bits on the GPU: rows stored and read back bit by bit, attention over it against plain 64-bit definitions."""
import math

import numpy as np
import pytest

import block_util as bu
from gpu_util import dev_bf16, host_f64, say
from synth_inputs import bf16_bits_to_f64, normal_bf16

pytestmark = pytest.mark.gpu

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def rounded(x):
    """x [..., 32 n] float64 -> (values, scale bytes) of the format, by its definition."""
    g = x.reshape(x.shape[:-1] + (-1, 32))
    most = np.abs(g).max(-1)
    e = np.full(most.shape, -125)
    for exponent in range(-125, 127):
        e[most >= 7.0 * 2.0 ** exponent] = exponent + 1
    y = np.abs(g) / 2.0 ** e[..., None]
    d = np.abs(y[..., None] - LEVELS)
    # the nearest code, of two equally near the even one
    code = np.where(d == d.min(-1, keepdims=True), np.arange(8) % 2, 2).argmin(-1)
    return (np.sign(g) * LEVELS[code] * 2.0 ** e[..., None]).reshape(x.shape), (e + 127).astype(np.uint8)


def random_cache(sp, B, N, H, D, salt=0):
    """(cache, k, v): a cache of random rows and the numbers it stands for, in 64 bits."""
    bits = [normal_bf16((B, N, H, D), 33, t, salt) for t in "kv"]
    cache = sp.KvCache4.empty(B, N, H, D)
    sp.slimpipe_attn_kv4_store(dev_bf16(bits[0]), dev_bf16(bits[1]), cache, 0)
    return cache, rounded(bf16_bits_to_f64(bits[0]))[0], rounded(bf16_bits_to_f64(bits[1]))[0]


def test_every_bf16_in_a_group_of_each_magnitude(sp):
    """Every finite bf16 value of 16 binades beside a largest element that decides the scale: all codes, all ties."""
    import torch
    say("kv4 store, all values")
    groups = []
    for top in (1.0, 1.5, 1.75, 1.7421875, 1.9921875, 6.0, 7.0, 2.0 ** -20, 2.0 ** 100):
        mant = np.arange(128) / 128.0 + 1.0
        vals = np.concatenate([mant * top * 2.0 ** -i for i in range(0, 8)])
        vals = bf16_bits_to_f64((np.float32(vals).view(np.uint32) >> 16).astype(np.uint16))
        vals = vals[vals <= top]
        vals = np.concatenate([vals, -vals])
        vals = np.concatenate([vals, np.zeros(-len(vals) % 31)]).reshape(-1, 31)
        groups.append(np.concatenate([vals, np.full((len(vals), 1), top)], 1))
    x = np.concatenate(groups)
    x = x[:len(x) // 4 * 4].reshape(1, -1, 1, 128)
    dev = torch.from_numpy(x).to("cuda").to(torch.bfloat16)
    assert np.array_equal(host_f64(dev), x)
    cache = sp.KvCache4.empty(1, x.shape[1], 1, 128)
    sp.slimpipe_attn_kv4_store(dev, -dev, cache, 0)
    want, scales = rounded(x)
    k, v = sp.slimpipe_attn_kv4_load(cache, 0, x.shape[1])
    assert np.array_equal(cache.k_scales.cpu().numpy(), scales)
    assert np.array_equal(host_f64(k), want) and np.array_equal(host_f64(v), -want)


def test_extreme_groups(sp):
    """Zeros, subnormal and largest magnitudes, an infinity, a NaN: only the group that holds one is not finite."""
    import torch
    x = torch.zeros((1, 6, 1, 64), device="cuda", dtype=torch.bfloat16)
    x[0, 1] = 2.0 ** -133
    x[0, 2] = torch.finfo(torch.bfloat16).max
    x[0, 3, 0, 5] = float("inf")
    x[0, 4, 0, 40] = float("nan")
    x[0, 5] = 2.0 ** -125 * 0.75
    cache = sp.KvCache4.empty(1, 6, 1, 64)
    sp.slimpipe_attn_kv4_store(x, x, cache, 0)
    k, _ = sp.slimpipe_attn_kv4_load(cache, 0, 6)
    got = host_f64(k)
    assert (got[0, 0] == 0).all() and (got[0, 1] == 0).all()
    assert np.isinf(got[0, 2]).all()                     # the nearest code is 4 times 2^126
    assert np.isnan(got[0, 3, 0, :32]).all() and (got[0, 3, 0, 32:] == 0).all()
    assert np.isnan(got[0, 4, 0, 32:]).all() and (got[0, 4, 0, :32] == 0).all()
    assert (got[0, 5] == 2.0 ** -125).all()              # 0.75 is as near to 0.5 as to 1: the even code


@pytest.mark.parametrize("B,N,H,D,s,at", [(1, 40, 1, 128, 1, 39), (3, 100, 2, 64, 17, 20), (2, 300, 5, 128, 133, 0), (2, 9, 3, 64, 9, 0)])
def test_store_writes_its_rows_alone(sp, B, N, H, D, s, at):
    import torch
    bits = normal_bf16((B, s, H, D), 34, "k"), normal_bf16((B, s, H, D), 34, "v")
    wide = torch.zeros((B, s, 3 * H, D), device="cuda", dtype=torch.bfloat16)
    k, v = wide[:, :, :H], wide[:, :, 2 * H:]
    k.copy_(dev_bf16(bits[0]))
    v.copy_(dev_bf16(bits[1]))
    cache = sp.KvCache4(*(x.fill_(0x55) for x in sp.KvCache4.empty(B, N, H, D)))
    sp.slimpipe_attn_kv4_store(k, v, cache, at)
    for x in cache:
        assert (x[:, :at] == 0x55).all() and (x[:, at + s:] == 0x55).all()
    want = [rounded(bf16_bits_to_f64(b)) for b in bits]
    assert np.array_equal(cache.k_scales[:, at:at + s].cpu().numpy(), want[0][1])
    got = sp.slimpipe_attn_kv4_load(cache, at, at + s)
    assert np.array_equal(host_f64(got[0]), want[0][0]) and np.array_equal(host_f64(got[1]), want[1][0])
    # the same cache with heads ahead of rows in memory
    turned = sp.KvCache4(*(x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in sp.KvCache4.empty(B, N, H, D)))
    sp.slimpipe_attn_kv4_store(k, v, turned, at)
    again = sp.slimpipe_attn_kv4_load(turned, at, at + s)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


# batch, rows, offset, heads, kv heads, head_dim, causal, (kv_begin, kv_end) or None
SHAPES = [
    (1, 1, 0, 1, 1, 128, True, None),
    (2, 1, 300, 8, 1, 64, True, None),
    (1, 1, 5000, 8, 1, 128, True, None),               # tokens: keys cut into parts
    (3, 4, 997, 8, 1, 128, True, None),                # 32 rows of a kv head, the most of a token call
    (2, 11, 700, 9, 3, 128, True, None),               # 33
    (1, 33, 0, 4, 4, 64, True, None),
    (2, 257, 1791, 6, 2, 64, True, None),
    (1, 300, 3700, 3, 1, 128, True, None),             # a slice, keys cut into parts
    (1, 200, 900, 2, 2, 128, False, None),
    (1, 2, 900, 4, 4, 64, False, (3, 890)),
    (2, 130, 400, 4, 1, 128, True, (100, 480)),
    (1, 130, 400, 4, 1, 64, True, (450, 500)),         # early rows see nothing
    (1, 3, 400, 4, 1, 64, True, (402, 403)),
    (1, 3, 400, 4, 1, 128, True, (200, 200)),
    (1, 50, 400, 4, 1, 128, True, (450, 450)),
]


@pytest.mark.parametrize("case", SHAPES)
def test_forward(sp, case):
    B, s, off, Hq, Hkv, D, causal, rng_ = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("kv4 forward %r" % (case,))
    cache, k, v = random_cache(sp, B, N, Hkv, D, salt=s)
    bits = normal_bf16((B, s, Hq, D), 33, "q", s)
    key = np.arange(N)
    see = (key >= begin) & (key < end) & ((key <= (off + np.arange(s))[:, None]) | (not causal))
    see = np.broadcast_to(see, (B, Hq, s, N))
    for dtype in (sp.BF16, sp.F32):
        r = bu.Reference(bf16_bits_to_f64(bits), k, v, see, 1 / math.sqrt(D), dtype == sp.BF16)
        out, lse = sp.slimpipe_attn_fwd_kv4(dev_bf16(bits), cache, off, begin, end, causal, out_dtype=dtype)
        bu.check("out", host_f64(out), r.out, r.out_tol)
        bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


@pytest.mark.parametrize("s", [2, 140])
def test_layouts_and_unseen_keys(sp, s):
    """Strided heads, a cache of another layout with NaN scales behind the last seen key: the same bits."""
    import torch
    B, off, Hq, Hkv, D = 2, 620, 4, 2, 128
    N = off + s
    cache, _, _ = random_cache(sp, B, N, Hkv, D)
    q = dev_bf16(normal_bf16((B, s, Hq, D), 33, "q"))
    out, lse = sp.slimpipe_attn_fwd_kv4(q, cache, off, 7, N)
    bigger = sp.KvCache4(*(x.fill_(0xff).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in sp.KvCache4.empty(B, N + 100, Hkv, D)))
    for x, y in zip(bigger, cache):
        x[:, 7:N] = y[:, 7:]
    wide = torch.zeros((B, s, Hq + 3, D), device="cuda", dtype=torch.bfloat16)
    wide[:, :, 1:1 + Hq] = q
    o2 = torch.zeros((B, s, 2 * Hq, D), device="cuda", dtype=torch.bfloat16)[:, :, Hq:]
    _, l2 = sp.slimpipe_attn_fwd_kv4(wide[:, :, 1:1 + Hq], bigger, off, 7, N + 100, out=o2, lse=torch.empty_like(lse))
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_old_prefix_in_4_bits_new_keys_in_bf16(sp):
    """As it is used: the prompt in 4 bits, what came since in bf16, the two folded by the merge; and sparse attention over the part in bf16."""
    B, s, old, Hq, Hkv, D, L = 1, 40, 700, 8, 2, 128, 64
    N, off = 1024, 1024 - 40
    cache, k4, v4 = random_cache(sp, B, old, Hkv, D)
    bits = {t: normal_bf16((B, n, H, D), 35, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv))}
    dev, ref = {t: dev_bf16(x) for t, x in bits.items()}, {t: bf16_bits_to_f64(x) for t, x in bits.items()}
    a = sp.slimpipe_attn_fwd_kv4(dev["q"], cache, off, 0, old, out_dtype=sp.F32)
    means = sp.slimpipe_attn_block_means(dev["k"], 0, N, L)
    index = sp.slimpipe_attn_block_select(dev["q"], means, off, old, N, L, 4)
    c = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], index, off, old, N, L, out_dtype=sp.F32)
    out, lse = sp.slimpipe_attn_merge([a[0], c[0]], [a[1], c[1]])
    k, v = ref["k"].copy(), ref["v"].copy()
    k[:, :old], v[:, :old] = k4, v4
    see = bu.visible(index.cpu().numpy(), off, old, N, L, True, N)
    see[..., :old] = True
    r = bu.Reference(ref["q"], k, v, see, 1 / math.sqrt(D))
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


def test_tokens_as_they_come_streams_and_graph(sp):
    """Tokens stored and attended to one by one, eagerly, on another stream and from a graph that is replayed with other rows."""
    import torch
    B, Hq, Hkv, D, N = 2, 8, 2, 64, 400
    rows = [dev_bf16(normal_bf16((B, N, H, D), 36, t)) for t, H in (("q", Hq), ("k", Hkv), ("v", Hkv))]

    def token(cache, t, ws=None):
        q, k, v = (x[:, t:t + 1] for x in rows)
        sp.slimpipe_attn_kv4_store(k, v, cache, t)
        return sp.slimpipe_attn_fwd_kv4(q, cache, t, 0, t + 1, workspace=ws)
    whole = sp.KvCache4.empty(B, N, Hkv, D)
    sp.slimpipe_attn_kv4_store(rows[1], rows[2], whole, 0)
    cache = sp.KvCache4.empty(B, N, Hkv, D)
    sp.slimpipe_attn_kv4_store(rows[1][:, :390], rows[2][:, :390], cache, 0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    eager = []
    with torch.cuda.stream(side):
        for t in range(390, N):
            eager.append(token(cache, t))
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(cache, whole))
    # a captured step over a fixed range, replayed with new rows in its buffers
    buf = [x[:, 390:391].clone() for x in rows]
    sp.slimpipe_attn_init()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sp.slimpipe_attn_kv4_store(buf[1], buf[2], cache, 390)
        got = sp.slimpipe_attn_fwd_kv4(buf[0], cache, 390, 0, 391)
    for t in (390, 391, 390):
        for x, y in zip(buf, rows):
            x.copy_(y[:, t:t + 1])
        graph.replay()
        torch.cuda.synchronize()
        sp.slimpipe_attn_kv4_store(buf[1], buf[2], cache, 390)
        want = sp.slimpipe_attn_fwd_kv4(buf[0], cache, 390, 0, 391)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        if t == 390:
            assert torch.equal(got[0], eager[0][0])
