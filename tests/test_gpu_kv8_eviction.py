"""Eviction from the cache in 8 bits on the GPU: sums of attention weights against 64 bits, the choice of rows index by index, the move bit by bit, and
all of it as it is used."""
import math

import numpy as np
import pytest

import kv8_util as ku
from gpu_util import dev_bf16, host_f64, say
from synth_inputs import bf16_bits_to_f64, normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def filled(sp, B, N, H, D, L, salt=0, factor=None):
    """(cache, k, v): a cache of random rows and the numbers it stands for."""
    import torch
    rows = [bf16_bits_to_f64(normal_bf16((B, N, H, D), 53, t, salt)) for t in "kv"]
    if factor is not None:
        rows = [x * factor for x in rows]
    dev = [torch.from_numpy(x).to(torch.bfloat16).cuda() for x in rows]
    cache = sp.KvCache8.empty(B, N, H, D, L)
    sp.slimpipe_attn_kv8_store(dev[0], dev[1], cache, 0)
    return (cache,) + tuple(ku.Cache(B, H, D, L).append(host_f64(x)) for x in dev)


# ------------------------------------------------------------------------------------------ sums of weights

# batch, rows, offset, heads, kv heads, head_dim, causal, (kv_begin, kv_end) or None, block
SHAPES = [
    (1, 1, 0, 1, 1, 128, True, None, 16),
    (2, 1, 300, 8, 1, 64, True, None, 64),
    (1, 1, 5000, 8, 1, 128, True, None, 128),
    (3, 4, 997, 8, 1, 128, True, None, 32),            # 32 rows of a kv head, the most of a token call
    (1, 2, 3000, 12, 4, 64, True, None, 16),           # four heads a workgroup
    (2, 11, 700, 9, 3, 128, True, None, 256),          # 33 rows: tiles over several heads
    (1, 33, 0, 4, 4, 64, True, None, 64),
    (2, 257, 1791, 6, 2, 64, True, None, 16),
    (1, 300, 3700, 3, 1, 128, True, None, 128),
    (1, 700, 2900, 8, 2, 128, True, None, 64),
    (1, 1500, 0, 8, 1, 64, True, None, 64),            # keys after keys that fewer rows see
    (1, 200, 900, 2, 2, 128, False, None, 32),
    (1, 2, 900, 4, 4, 64, False, (3, 890), 32),
    (2, 130, 400, 4, 1, 128, True, (100, 480), 16),
    (1, 130, 400, 4, 1, 64, True, (450, 500), 64),     # early rows see nothing
    (1, 3, 400, 4, 1, 128, True, (200, 200), 64),
    (1, 40, 100, 4, 1, 128, True, (0, 700), 64),       # keys behind the last row
]


@pytest.mark.parametrize("case", SHAPES)
def test_weights(sp, case):
    import torch
    B, s, off, Hq, Hkv, D, causal, rng_, L = case
    begin, end = rng_ or (0, off + s)
    N = max(off + s, end) + 5
    say("kv8 weights %r" % (case,))
    cache, k, _ = filled(sp, B, N, Hkv, D, L, salt=s)
    bits = normal_bf16((B, s, Hq, D), 53, "q", s)
    q, scale = bf16_bits_to_f64(bits), 1 / math.sqrt(D)
    key = np.arange(N)
    see = (key >= begin) & (key < end) & ((key <= (off + np.arange(s))[:, None]) | (not causal))
    x = np.where(see, scale * np.einsum("bshd,bnhd->bhsn", q, np.repeat(k.values, Hq // Hkv, 2)), -np.inf)
    with np.errstate(divide="ignore"):
        top = np.max(x, -1, keepdims=True, initial=-np.inf)
        lse = np.where(np.isinf(top), 0, top) + np.log(np.exp(x - np.where(np.isinf(top), 0, top)).sum(-1, keepdims=True))
    p = np.exp(x - np.where(np.isinf(lse), 0.0, lse))
    lse32 = np.ascontiguousarray(np.float32(lse[..., 0]))
    want = p.reshape(B, Hkv, -1, N).sum(2)
    before = np.float32(np.random.RandomState(3).rand(B, Hkv, N))
    dev = torch.from_numpy(lse32).cuda(), torch.from_numpy(before).cuda()
    args = (dev_bf16(bits), cache, dev[0], off, begin, end, causal)
    got = sp.slimpipe_attn_kv8_weights(*args)
    # a score of D products and its lse are off by at most D 2^-24 sum |q k| and 2^-24 |lse| (its rounding here), the exponential by 2^-20; so is each term
    # of the sum, and the sum by 2^-24 a term
    size = scale * np.abs(q).sum(-1).max() * np.abs(k.values).max()
    rel = D * 2.0 ** -24 * size + 2.0 ** -23 * (np.abs(np.where(np.isinf(lse), 0.0, lse)).max() + np.abs(np.where(np.isinf(x), 0.0, x)).max()) + 2.0 ** -20
    rel += s * Hq // Hkv * 2.0 ** -24
    inside = (key >= begin) & (key < end)
    assert (np.abs(host_f64(got) - np.where(inside, want, 0.0)) <= rel * want + 1e-30).all()
    # added to decayed sums, other entries left alone; also in place; the same bits again
    out = torch.full((B, Hkv, N), -5.0, device="cuda")
    got2 = sp.slimpipe_attn_kv8_weights(*args, weights=out, previous=dev[1], decay=0.75)
    total = want + 0.75 * before
    assert (np.abs(host_f64(got2) - total)[..., inside] <= (rel * want + 2.0 ** -23 * total)[..., inside]).all()
    assert (got2[..., ~torch.from_numpy(inside).cuda()] == -5.0).all()
    place = dev[1].clone()
    sp.slimpipe_attn_kv8_weights(*args, weights=place, previous=place, decay=0.75)
    assert torch.equal(place[..., begin:end], got2[..., begin:end]) and torch.equal(place[..., end:], dev[1][..., end:])
    assert torch.equal(sp.slimpipe_attn_kv8_weights(*args), got)


@pytest.mark.parametrize("s", [3, 90])
def test_weights_of_rows_that_saw_nothing_and_unseen_keys(sp, s):
    """Rows with lse -infinity add nothing; keys that no row sees hold NaN and get none; strided queries."""
    import torch
    B, off, Hq, Hkv, D, L = 1, 200, 4, 2, 128, 16
    N = off + s
    cache, _, _ = filled(sp, B, N + 40, Hkv, D, L)
    q = dev_bf16(normal_bf16((B, s, Hq, D), 53, "q"))
    _, lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, 0, N)
    want = sp.slimpipe_attn_kv8_weights(q, cache, lse, off, 0, N)
    assert abs(float(want.sum()) - s * Hq) <= s * Hq * 2.0 ** -10      # (every row's weights sum to 1)
    cache.k_codes[:, N:] = 0x7f
    wide = torch.zeros((B, s, Hq + 3, D), device="cuda", dtype=torch.bfloat16)
    wide[:, :, 1:1 + Hq] = q
    again = sp.slimpipe_attn_kv8_weights(wide[:, :, 1:1 + Hq], cache, lse, off, 0, N + 30)
    assert (again[..., :N] - want[..., :N]).abs().max() <= s * Hq * 2.0 ** -22 and (again[..., N:] == 0).all()
    part = lse.clone()
    part[:, 1] = -math.inf
    part[:, 3] = -math.inf
    half = sp.slimpipe_attn_kv8_weights(q, cache, part, off, 0, N)
    assert abs(float(half.sum()) - s * Hq / 2) <= s * Hq * 2.0 ** -10


# ------------------------------------------------------------------------------------------ the choice

def chosen(w, rows, keep, recent):
    """w [B, H, N] -> index by a stable sort: NaN last, zeros alike."""
    x = w[..., :rows - recent].astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    nan = np.isnan(w[..., :rows - recent])
    order = np.lexsort((np.broadcast_to(np.arange(rows - recent), x.shape), -x, nan), axis=-1)[..., :keep - recent]
    late = np.broadcast_to(np.arange(rows - recent, rows), w.shape[:2] + (recent,))
    return np.concatenate([np.sort(order, -1), late], -1)


def spread(kind, shape, seed):
    g = np.random.RandomState(seed)
    x = np.exp(3 * g.randn(*shape)).astype(np.float32)
    if kind == "equal":
        x[:] = 0.25
    elif kind == "few":
        x = (g.randint(0, 3, shape) / 2).astype(np.float32)
    elif kind == "near":                                     # neighbours in 32 bits: the last digits decide
        x = (1 + g.randint(0, 40, shape) * 2.0 ** -23).astype(np.float32)
    elif kind == "odd":
        x = (g.randn(*shape) * 10.0 ** g.randint(-38, 38, shape)).astype(np.float32)
        for v in (np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45):
            x[g.rand(*shape) < 0.08] = v
    return x


@pytest.mark.parametrize("kind", ["any", "equal", "few", "near", "odd"])
@pytest.mark.parametrize("B,H,N,rows,keep,recent", [(1, 1, 1, 1, 1, 0), (1, 2, 70, 64, 1, 1), (2, 3, 1024, 1024, 1024, 7), (1, 1, 1025, 1025, 1, 0),
                                                    (2, 1, 5000, 4238, 2119, 337), (1, 4, 9000, 8193, 8000, 0), (1, 2, 20000, 20000, 500, 500),
                                                    (3, 2, 33333, 33331, 12345, 100), (1, 3, 140001, 140001, 33000, 1024), (1, 2, 40000, 40000, 40000, 7),
                                                    (1, 2, 40000, 39999, 500, 500), (2, 1, 33000, 33000, 33000, 33000), (1, 1, 600000, 599999, 3, 1),
                                                    (2, 2, 16384, 16384, 9000, 50), (2, 2, 17000, 16385, 9000, 0), (1, 3, 30000, 28000, 27000, 900)])
def test_keep(sp, kind, B, H, N, rows, keep, recent):
    import torch
    say("kv8 keep %s %r" % (kind, (B, H, N, rows, keep, recent)))
    w = spread(kind, (B, H, N), N + keep)
    index = sp.slimpipe_attn_kv8_keep(torch.from_numpy(w).cuda(), rows, keep, recent)
    assert np.array_equal(index.cpu().numpy(), chosen(w, rows, keep, recent))


# ------------------------------------------------------------------------------------------ the move

@pytest.mark.parametrize("B,N,H,D,L,keep", [(1, 5, 1, 64, 16, 1), (2, 300, 3, 128, 16, 133), (1, 700, 4, 64, 64, 350), (2, 600, 2, 128, 128, 257), (1, 1100, 5, 64, 256, 900)])
def test_gather(sp, B, N, H, D, L, keep):
    import torch
    say("kv8 gather %r" % ((B, N, H, D, L, keep),))
    # scales differ from block to block, by up to 2^12
    factor = 2.0 ** np.repeat(np.random.RandomState(1).randint(0, 13, -(-N // L)), L)[:N][None, :, None, None]
    cache, k, v = filled(sp, B, N, H, D, L, factor=factor)
    index = np.sort(np.random.RandomState(2).rand(B, H, N).argsort(-1)[..., :keep], -1).astype(np.int32)
    w = np.random.RandomState(3).rand(B, H, N).astype(np.float32)
    M = keep + 70
    kept = sp.KvCache8(*(x.fill_(0x55) for x in sp.KvCache8.empty(B, M, H, D, L)[:4]), L)
    sums = torch.full((B, H, M), -5.0, device="cuda")
    assert sp.slimpipe_attn_kv8_gather(cache, torch.from_numpy(index).cuda(), kept, torch.from_numpy(w).cuda(), sums) is kept
    got = sp.slimpipe_attn_kv8_load(kept, 0, keep)
    blocks = -(-keep // L)
    for x, y, codes, scales in zip((k, v), got, (kept.k_codes, kept.v_codes), (kept.k_scales, kept.v_scales)):
        units = np.zeros((B, blocks, H))
        want = np.zeros((B, keep, H, D))
        for h in range(H):
            for b in range(B):
                rows = index[b, h]
                u = x.units[b, rows // L, h]
                units[b, :, h] = [u[j * L:(j + 1) * L].max() for j in range(blocks)]
                want[b, :, h] = ku.round_to(x.values[b, rows, h], np.repeat(units[b, :, h], L)[:keep, None])
        assert np.array_equal(host_f64(y), want)
        assert np.array_equal(scales[:, :blocks].cpu().numpy(), (np.log2(units) + 127).astype(np.uint8))
        assert (scales[:, blocks:] == 0x55).all() and (codes[:, keep:] == 0x55).all()
    assert np.array_equal(sums[..., :keep].cpu().numpy(), np.take_along_axis(w, index.astype(np.int64), 2)) and (sums[..., keep:] == -5.0).all()


def test_gather_rows_twice_and_entries_that_are_no_row(sp):
    import torch
    cache, k, _ = filled(sp, 1, 40, 1, 64, 16)
    index = torch.tensor([[[3, 3, -1, 39, 40, 2 ** 31 - 1, -2 ** 31, 0]]], device="cuda", dtype=torch.int32)
    kept = sp.slimpipe_attn_kv8_gather(cache, index, sp.KvCache8.empty(1, 8, 1, 64, 16))
    got = host_f64(sp.slimpipe_attn_kv8_load(kept, 0, 8)[0])[0, :, 0]
    u = max(k.units[0, j, 0] for j in (0, 2))
    want = ku.round_to(np.where(np.array([1, 1, 0, 1, 0, 0, 0, 1])[:, None] > 0, k.values[0, [3, 3, 0, 39, 0, 0, 0, 0], 0], 0.0), u)
    assert np.array_equal(got, want)
    empty = sp.slimpipe_attn_kv8_gather(cache, index[..., :0].contiguous(), kept)
    assert empty is kept and np.array_equal(host_f64(sp.slimpipe_attn_kv8_load(kept, 0, 8)[0])[0, :, 0], want)


# ------------------------------------------------------------------------------------------ as it is used

def test_prompt_eviction_tokens(sp):
    """A prompt in slices, normalised, rotated, appended and attended to; its rows weighed, half of them kept; tokens go on behind them, rotated by their own
    positions, over a cache of fewer rows.  The tokens' attention against 64 bits over the rows that are there."""
    import torch
    B, Hq, Hkv, D, L, n, slices, recent = 2, 8, 2, 64, 32, 600, 3, 40
    g = torch.Generator(device="cuda").manual_seed(77)
    x = torch.randn((B, n + 4, Hq + 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    wq, wk = 1.0 + 0.2 * torch.randn((2, D), generator=g, device="cuda")
    freq = torch.pow(10000.0, -2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    parts = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    cache, sums = sp.KvCache8.empty(B, n, Hkv, D, L), None
    step = n // slices
    for i in range(slices):
        r = slice(i * step, (i + 1) * step)
        q, k = sp.slimpipe_attn_norm_rotate(parts[0][:, r], parts[1][:, r], wq, wk, freq, r.start)
        sp.slimpipe_attn_kv8_store(k, parts[2][:, r].contiguous(), cache, r.start)
        _, lse = sp.slimpipe_attn_fwd_kv8(q, cache, r.start, 0, r.stop)
        sums = sp.slimpipe_attn_kv8_weights(q, cache, lse, r.start, 0, r.stop, weights=sums, previous=sums)
    assert (sums.sum((1, 2)) - n * Hq).abs().max() <= n * Hq * 2.0 ** -9
    keep = n // 2
    index = sp.slimpipe_attn_kv8_keep(sums, n, keep, recent)
    assert np.array_equal(index.cpu().numpy(), chosen(sums.cpu().numpy(), n, keep, recent))
    small, small_sums = sp.KvCache8.empty(B, keep + 4, Hkv, D, L), torch.zeros((B, Hkv, keep + 4), device="cuda")
    sp.slimpipe_attn_kv8_gather(cache, index, small, sums, small_sums)
    for t in range(4):
        r = slice(n + t, n + t + 1)
        q, k = sp.slimpipe_attn_norm_rotate(parts[0][:, r], parts[1][:, r], wq, wk, freq, n + t)
        sp.slimpipe_attn_kv8_store(k, parts[2][:, r].contiguous(), small, keep + t)
        out, lse = sp.slimpipe_attn_fwd_kv8(q, small, keep + t, 0, keep + t + 1, out_dtype=sp.F32)
        before = float(small_sums.sum())
        sp.slimpipe_attn_kv8_weights(q, small, lse, keep + t, 0, keep + t + 1, weights=small_sums, previous=small_sums)
        # (each of the B Hq rows adds 1; sums of some thousands in 32 bits)
        assert abs(float(small_sums.sum()) - before - B * Hq) <= 0.05
        kk, vv = (np.repeat(host_f64(y), Hq // Hkv, 2) for y in sp.slimpipe_attn_kv8_load(small, 0, keep + t + 1))
        s = np.einsum("bhd,bnhd->bhn", host_f64(q)[:, 0], kk) / math.sqrt(D)
        p = np.exp(s - s.max(-1, keepdims=True))
        total = p.sum(-1, keepdims=True)
        want = np.einsum("bhn,bnhd->bhd", p / total, vv)
        # (probabilities rounded to bf16: 2^-8 of the average of |v|)
        assert (np.abs(host_f64(out)[:, 0] - want) <= 2.0 ** -8 * np.einsum("bhn,bnhd->bhd", p / total, np.abs(vv)) + 1e-4).all()
        assert np.abs(host_f64(lse)[:, :, 0] - (s.max(-1) + np.log(total[..., 0]))).max() <= 1e-4


def test_captured(sp):
    """The three calls in a graph, replayed on other inputs, against eager calls."""
    import torch
    sp.slimpipe_attn_init()
    for s in (2, 100):
        B, Hq, Hkv, D, L, N, keep = 2, 8, 2, 128, 64, 700, 300
        cache, _, _ = filled(sp, B, N, Hkv, D, L)
        q = dev_bf16(normal_bf16((B, s, Hq, D), 53, "q"))
        lse = sp.slimpipe_attn_fwd_kv8(q, cache, N - s, 0, N)[1]
        sums, old = torch.zeros((B, Hkv, N), device="cuda"), torch.rand((B, Hkv, N), device="cuda")
        index = torch.zeros((B, Hkv, keep), device="cuda", dtype=torch.int32)
        kept, kept_sums = sp.KvCache8.empty(B, keep, Hkv, D, L), torch.zeros((B, Hkv, keep), device="cuda")
        ws = [torch.empty(k, device="cuda", dtype=torch.uint8) for k in (sp.slimpipe_attn_kv8_weights_workspace_bytes(q, cache, N - s, 0, N),
                                                                        sp.slimpipe_attn_kv8_keep_workspace_bytes(sums, N, keep))]

        def calls():
            sp.slimpipe_attn_kv8_weights(q, cache, lse, N - s, 0, N, weights=sums, previous=old, decay=0.5, workspace=ws[0])
            sp.slimpipe_attn_kv8_keep(sums, N, keep, 20, index=index, workspace=ws[1])
            sp.slimpipe_attn_kv8_gather(cache, index, kept, sums, kept_sums)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for n in range(3):
            old.uniform_()
            lse.add_(0.1 * n)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (sums, index, kept_sums) + kept[:4]]
            calls()
            assert all(torch.equal(a, b) for a, b in zip(got, (sums, index, kept_sums) + kept[:4]))
