"""The key/value cache in 8 bits on the GPU: rows appended and read back bit by bit, attention over it against plain 64-bit definitions."""
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


def same(a, b):
    """(NaN in the same places)"""
    return np.array_equal(a, b, equal_nan=True)


def random_cache(sp, B, N, H, D, L, salt=0):
    """(cache, k, v): a cache of random rows and the numbers it stands for, in 64 bits."""
    bits = [normal_bf16((B, N, H, D), 43, t, salt) for t in "kv"]
    cache = sp.KvCache8.empty(B, N, H, D, L)
    sp.slimpipe_attn_kv8_store(dev_bf16(bits[0]), dev_bf16(bits[1]), cache, 0)
    return (cache,) + tuple(ku.Cache(B, H, D, L).append(bf16_bits_to_f64(b)).values for b in bits)


def test_every_bf16_in_a_block_of_each_magnitude(sp):
    """Every finite bf16 value of 20 binades beside a largest element that decides the scale: all codes, all ties, both signs."""
    import torch
    say("kv8 store, all values")
    blocks = []
    for top in (1.0, 1.5, 1.75, 1.7578125, 1.9921875, 448.0, 450.0, 2.0 ** -20, 1.75 * 2.0 ** 100, 2.0 ** 127 * 1.9921875, 2.0 ** -101, 2.0 ** -106):
        mant = np.arange(128) / 128.0 + 1.0
        vals = np.concatenate([mant * top * 2.0 ** -i for i in range(0, 20)])
        vals = vals[vals < 2.0 ** 128]
        vals = bf16_bits_to_f64((np.float32(vals).view(np.uint32) >> 16).astype(np.uint16))
        vals = vals[(vals <= top) & (vals > 0)]
        vals = np.concatenate([vals, -vals])
        vals = np.concatenate([vals, np.zeros(-len(vals) % (16 * 64 - 1))]).reshape(-1, 16 * 64 - 1)
        blocks.append(np.concatenate([vals, np.full((len(vals), 1), top)], 1).reshape(-1, 64))
    x = np.concatenate(blocks).reshape(1, -1, 1, 64)
    dev = torch.from_numpy(x).to("cuda").to(torch.bfloat16)
    assert np.array_equal(host_f64(dev), x)
    cache = sp.KvCache8.empty(1, x.shape[1], 1, 64, 16)
    sp.slimpipe_attn_kv8_store(dev, -dev, cache, 0)
    want = ku.Cache(1, 1, 64, 16).append(x)
    k, v = sp.slimpipe_attn_kv8_load(cache, 0, x.shape[1])
    assert np.array_equal(cache.k_scales.cpu().numpy(), want.scales())
    values = np.where(want.values >= 2.0 ** 128, np.inf, np.where(want.values <= -2.0 ** 128, -np.inf, want.values))      # (past the largest bf16)
    for got, sign in ((k, 1), (v, -1)):
        off = host_f64(got) != sign * values
        assert not off.any(), list(zip(x[off][:8], host_f64(got)[off][:8], sign * values[off][:8]))


def test_values_that_are_not_finite_and_extremes(sp):
    """Zeros, subnormal and largest magnitudes, infinities, NaN of both signs: only the element itself is not finite."""
    import torch
    x = torch.zeros((1, 96, 1, 64), device="cuda", dtype=torch.bfloat16)
    x[0, 16:32] = 2.0 ** -133
    x[0, 32:48] = torch.finfo(torch.bfloat16).max
    x[0, 48, 0, 5], x[0, 49, 0, 6], x[0, 50, 0, 7] = float("inf"), float("-inf"), 3.0
    x[0, 64, 0, 40], x[0, 65, 0, 41] = float("nan"), -float("nan")
    x[0, 80:] = 2.0 ** -112
    cache = sp.KvCache8.empty(1, 96, 1, 64, 16)
    sp.slimpipe_attn_kv8_store(x, -x, cache, 0)
    k, v = sp.slimpipe_attn_kv8_load(cache, 0, 96)
    want = ku.Cache(1, 1, 64, 16).append(host_f64(x))
    values = np.where(np.abs(want.values) >= 2.0 ** 128, np.inf, want.values)                            # (past the largest bf16)
    assert same(host_f64(k), values) and same(host_f64(v), -values)
    assert np.array_equal(cache.k_scales.cpu().numpy(), want.scales())
    assert np.isnan(want.values).sum() == 4


# batch, capacity, heads, head_dim, block, rows before, rows
STORES = [(1, 40, 1, 128, 16, 39, 1), (3, 100, 2, 64, 32, 20, 17), (2, 300, 5, 128, 64, 0, 133), (2, 9, 3, 64, 16, 0, 9), (1, 700, 3, 128, 128, 5, 600),
          (2, 1100, 2, 64, 128, 100, 900), (1, 1200, 2, 128, 256, 300, 801), (1, 1200, 4, 64, 256, 1, 1199), (1, 64, 40, 128, 16, 17, 47)]


@pytest.mark.parametrize("B,N,H,D,L,at,s", STORES)
def test_store_behind_rows_that_are_there(sp, B, N, H, D, L, at, s):
    """Rows larger and smaller than those before: scales grow or stay, earlier rows move with them; codes of other rows stay as they were."""
    import torch
    say("kv8 store %r" % ((B, N, H, D, L, at, s),))
    bits = [bf16_bits_to_f64(normal_bf16((B, at + s, H, D), 44, t)) for t in "kv"]
    rows = []
    for x, grow in zip(bits, (3.0, 0.01)):
        # (each head by another factor: in some of them the scale of the first block grows, in some it stays)
        x = x.copy()
        x[:, at:] *= grow * 2.0 ** (np.arange(H) % 3)[None, None, :, None]
        rows.append(torch.from_numpy(x).to(torch.bfloat16).cuda())
    wide = torch.zeros((B, at + s, 3 * H, D), device="cuda", dtype=torch.bfloat16)
    k, v = wide[:, :, :H], wide[:, :, 2 * H:]
    k.copy_(rows[0])
    v.copy_(rows[1])
    cache = sp.KvCache8(*(x.fill_(0x55) for x in sp.KvCache8.empty(B, N, H, D, L)[:4]), L)
    if at:
        sp.slimpipe_attn_kv8_store(k[:, :at], v[:, :at], cache, 0)
    sp.slimpipe_attn_kv8_store(k[:, at:], v[:, at:], cache, at)
    got = sp.slimpipe_attn_kv8_load(cache, 0, at + s)
    for x, y, scales, codes in zip(rows, got, (cache.k_scales, cache.v_scales), (cache.k_codes, cache.v_codes)):
        want = ku.Cache(B, H, D, L)
        if at:
            want.append(host_f64(x[:, :at]))
        want.append(host_f64(x[:, at:]))
        assert np.array_equal(host_f64(y), want.values)
        n = want.units.shape[1]
        assert np.array_equal(scales[:, :n].cpu().numpy(), want.scales())
        assert (scales[:, n:] == 0x55).all() and (codes[:, at + s:] == 0x55).all()
    # the same cache with heads ahead of rows in memory
    turned = sp.KvCache8(*(x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if x.dim() == 4 else x for x in sp.KvCache8.empty(B, N, H, D, L)[:4]), L)
    if at:
        sp.slimpipe_attn_kv8_store(k[:, :at], v[:, :at], turned, 0)
    sp.slimpipe_attn_kv8_store(k[:, at:], v[:, at:], turned, at)
    again = sp.slimpipe_attn_kv8_load(turned, 0, at + s)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


# batch, rows, offset, heads, kv heads, head_dim, causal, (kv_begin, kv_end) or None, block
SHAPES = [
    (1, 1, 0, 1, 1, 128, True, None, 16),
    (2, 1, 300, 8, 1, 64, True, None, 64),
    (1, 1, 5000, 8, 1, 128, True, None, 128),          # tokens: keys cut into parts
    (3, 4, 997, 8, 1, 128, True, None, 32),            # 32 rows of a kv head, the most of a token call
    (2, 11, 700, 9, 3, 128, True, None, 256),          # 33
    (1, 2, 3000, 12, 4, 64, True, None, 16),           # four heads a workgroup
    (2, 1, 1500, 4, 2, 128, True, None, 64),           # two
    (1, 33, 0, 4, 4, 64, True, None, 64),
    (2, 257, 1791, 6, 2, 64, True, None, 16),
    (1, 300, 3700, 3, 1, 128, True, None, 128),        # a slice, keys cut into parts
    (1, 700, 2900, 8, 2, 128, True, None, 64),
    (1, 200, 900, 2, 2, 128, False, None, 32),
    (8, 150, 2100, 8, 8, 64, True, None, 32),          # enough of it for workgroups of eight waves, one part and several
    (4, 300, 1000, 16, 16, 128, True, (500, 1300), 64),
    (3, 400, 1300, 9, 3, 64, False, None, 128),
    (1, 2, 900, 4, 4, 64, False, (3, 890), 32),
    (2, 130, 400, 4, 1, 128, True, (100, 480), 16),
    (1, 130, 400, 4, 1, 64, True, (450, 500), 64),     # early rows see nothing
    (1, 3, 400, 4, 1, 64, True, (402, 403), 64),
    (1, 3, 400, 4, 1, 128, True, (200, 200), 64),
    (1, 50, 400, 4, 1, 128, True, (450, 450), 64),
    (1, 48, 1306, 8, 2, 128, True, None, 64),          # few rows of a slice: ranges down to 128 keys
    (1, 60, 6000, 3, 1, 64, True, None, 16),
    (2, 500, 100, 4, 1, 128, True, None, 64),          # ranges that only late rows see
    (1, 130, 200, 4, 1, 128, True, (150, 330), 32),    # and rows before any of them
]


@pytest.mark.parametrize("case", SHAPES)
def test_forward(sp, case):
    B, s, off, Hq, Hkv, D, causal, rng_, L = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("kv8 forward %r" % (case,))
    cache, k, v = random_cache(sp, B, N, Hkv, D, L, salt=s)
    bits = normal_bf16((B, s, Hq, D), 43, "q", s)
    key = np.arange(N)
    see = (key >= begin) & (key < end) & ((key <= (off + np.arange(s))[:, None]) | (not causal))
    see = np.broadcast_to(see, (B, Hq, s, N))
    for dtype in (sp.BF16, sp.F32):
        r = bu.Reference(bf16_bits_to_f64(bits), k, v, see, 1 / math.sqrt(D), dtype == sp.BF16)
        out, lse = sp.slimpipe_attn_fwd_kv8(dev_bf16(bits), cache, off, begin, end, causal, out_dtype=dtype)
        bu.check("out", host_f64(out), r.out, r.out_tol)
        bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


def test_long_slice_with_and_without_room_for_a_copy(sp):
    """2200 rows of a kv head, the whole range and a piece of it: by a bf16 copy of the keys, and tile by tile where the workspace has no room for one."""
    import torch
    B, s, off, Hq, Hkv, D, L = 1, 1100, 333, 4, 2, 64, 32
    N = off + s
    cache, k, v = random_cache(sp, B, N, Hkv, D, L)
    bits = normal_bf16((B, s, Hq, D), 43, "q", 1)
    for begin, end in ((0, N), (301, 800)):
        key = np.arange(N)
        see = np.broadcast_to((key >= begin) & (key < end) & (key <= (off + np.arange(s))[:, None]), (B, Hq, s, N))
        r = bu.Reference(bf16_bits_to_f64(bits), k, v, see, 1 / math.sqrt(D))
        need = sp.slimpipe_attn_kv8_workspace_bytes(dev_bf16(bits), cache, off, begin, end)
        copy = 2 * B * (end - begin) * Hkv * D * 2
        assert need >= copy
        for room in (need, copy, copy - 256, 1 << 20, 0):
            ws = torch.empty(room, device="cuda", dtype=torch.uint8)
            out, lse = sp.slimpipe_attn_fwd_kv8(dev_bf16(bits), cache, off, begin, end, workspace=ws)
            bu.check("out", host_f64(out), r.out, r.out_tol)
            bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


@pytest.mark.parametrize("s", [2, 140, 520, 1100])
def test_layouts_and_unseen_keys(sp, s):
    """Strided heads, a cache of another layout with NaN codes and scales behind the last seen key and before the first: the same bits."""
    import torch
    B, off, Hq, Hkv, D, L = 2, 620, 4, 2, 128, 16
    N = off + s
    cache, _, _ = random_cache(sp, B, N, Hkv, D, L)
    q = dev_bf16(normal_bf16((B, s, Hq, D), 43, "q"))
    out, lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, 20, N)
    big = sp.KvCache8.empty(B, N + 100, Hkv, D, L)
    bigger = sp.KvCache8(*(x.fill_(0xff).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if x.dim() == 4 else x.fill_(0xff) for x in big[:4]), L)
    for x, y in zip(bigger[0:4:2], cache[0:4:2]):
        x[:, 20:N] = y[:, 20:]
    for x, y in zip(bigger[1:4:2], cache[1:4:2]):
        x[:, 1:y.shape[1]] = y[:, 1:]
    wide = torch.zeros((B, s, Hq + 3, D), device="cuda", dtype=torch.bfloat16)
    wide[:, :, 1:1 + Hq] = q
    o2 = torch.zeros((B, s, 2 * Hq, D), device="cuda", dtype=torch.bfloat16)[:, :, Hq:]
    _, l2 = sp.slimpipe_attn_fwd_kv8(wide[:, :, 1:1 + Hq], bigger, off, 20, N + 100, out=o2, lse=torch.empty_like(lse))
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_a_row_without_a_key_beside_rows_that_see_nan(sp):
    """Keys of the range hold NaN: rows that see them are NaN, a row that sees none has 0 and -infinity."""
    import torch
    for s, Hq in ((4, 2), (150, 2)):
        cache, _, _ = random_cache(sp, 1, 400, 1, 64, 16)
        x = torch.full((1, 400, 1, 64), float("nan"), device="cuda", dtype=torch.bfloat16)
        sp.slimpipe_attn_kv8_store(x, x, cache, 0)
        q = dev_bf16(normal_bf16((1, s, Hq, 64), 43, "q"))
        out, lse = sp.slimpipe_attn_fwd_kv8(q, cache, 100, 102, 400)
        assert (out[:, :2] == 0).all() and torch.isneginf(lse[..., :2]).all()
        assert torch.isnan(out[:, 2:].float()).all() and torch.isnan(lse[..., 2:]).all()


def test_old_prefix_in_8_bits_new_keys_in_bf16(sp):
    """The prompt in 8 bits, what came since in bf16, the two folded by the merge."""
    B, s, old, Hq, Hkv, D = 1, 40, 700, 8, 2, 128
    N, off = 1024, 1024 - 40
    cache, k8, v8 = random_cache(sp, B, old, Hkv, D, 64)
    bits = {t: normal_bf16((B, n, H, D), 45, t) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv))}
    dev, ref = {t: dev_bf16(x) for t, x in bits.items()}, {t: bf16_bits_to_f64(x) for t, x in bits.items()}
    a = sp.slimpipe_attn_fwd_kv8(dev["q"], cache, off, 0, old, out_dtype=sp.F32)
    c = sp.slimpipe_attn_fwd(dev["q"], dev["k"], dev["v"], off, old, N, out_dtype=sp.F32)
    out, lse = sp.slimpipe_attn_merge([a[0], c[0]], [a[1], c[1]])
    k, v = ref["k"].copy(), ref["v"].copy()
    k[:, :old], v[:, :old] = k8, v8
    see = np.broadcast_to(np.arange(N) <= (off + np.arange(s))[:, None], (B, Hq, s, N))
    r = bu.Reference(ref["q"], k, v, see, 1 / math.sqrt(D))
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


def test_tokens_as_they_come_streams_and_graph(sp):
    """Tokens appended and attended to one by one, eagerly, on another stream and from a graph that is replayed with other rows."""
    import torch
    B, Hq, Hkv, D, N, L = 2, 8, 2, 64, 400, 32
    rows = [dev_bf16(normal_bf16((B, N, H, D), 46, t)) for t, H in (("q", Hq), ("k", Hkv), ("v", Hkv))]

    def token(cache, t, ws=None):
        q, k, v = (x[:, t:t + 1] for x in rows)
        sp.slimpipe_attn_kv8_store(k, v, cache, t)
        return sp.slimpipe_attn_fwd_kv8(q, cache, t, 0, t + 1, workspace=ws)
    whole = ku.Cache(B, Hkv, D, L).append(host_f64(rows[1][:, :370]))
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(rows[1][:, :370], rows[2][:, :370], cache, 0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    eager = []
    with torch.cuda.stream(side):
        for t in range(370, N):
            eager.append(token(cache, t))
    side.synchronize()
    for t in range(370, N):
        whole.append(host_f64(rows[1][:, t:t + 1]))
    assert np.array_equal(host_f64(sp.slimpipe_attn_kv8_load(cache, 0, N)[0]), whole.values)
    assert np.array_equal(cache.k_scales.cpu().numpy(), whole.scales())
    # a captured step over a fixed range, replayed with new rows in its buffers
    buf = [x[:, 370:371].clone() for x in rows]
    sp.slimpipe_attn_init()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sp.slimpipe_attn_kv8_store(buf[1], buf[2], cache, 370)
        got = sp.slimpipe_attn_fwd_kv8(buf[0], cache, 370, 0, 371)
    for t in (370, 371, 370):
        for x, y in zip(buf, rows):
            x.copy_(y[:, t:t + 1])
        graph.replay()
        torch.cuda.synchronize()
        sp.slimpipe_attn_kv8_store(buf[1], buf[2], cache, 370)
        want = sp.slimpipe_attn_fwd_kv8(buf[0], cache, 370, 0, 371)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
