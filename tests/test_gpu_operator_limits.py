"""Sparse attention and the 4-bit cache where sizes, values and company are unusual: many rows and blocks, equal and tiny scores, values that are
not finite, offsets past 32 bits, two streams, two graphs on one workspace, and a training run over a sliced sequence."""
import math

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


def rows(shape, tag, salt=0):
    bits = normal_bf16(shape, 37, tag, salt)
    return dev_bf16(bits), bf16_bits_to_f64(bits)


def best_blocks(q, m, off, first, end, L, top_k, causal):
    """block_util.select, whole arrays at a time: q [B, s, Hq, D], m [B, Hkv, blocks, D]; blocks first .. end - 1 compete."""
    B, s, Hq, D = q.shape
    g = Hq // m.shape[1]
    index = np.full((B, Hq, s, top_k), -1)
    own = (off + np.arange(s)) // L
    for b in range(B):
        for h in range(Hq):
            score = q[b, :, h] @ m[b, h // g, first:end].T
            j = np.arange(first, end)[None]
            score = np.where(np.isnan(score), -np.inf, score)
            rank = np.argsort(np.argsort(np.where((j < own[:, None]) | (not causal), -score, np.nan), axis=1, kind="stable"), axis=1)
            forced = causal & (own >= first) & (own < end)
            take = (rank < (top_k - forced)[:, None]) & ((j < own[:, None]) | (not causal))
            take |= (j == own[:, None]) & forced[:, None]
            for r in range(s):
                n = j[0, take[r]]
                index[b, h, r, :len(n)] = n
    return index


# batch, rows, offset, heads, kv heads, head_dim, block, top_k, causal, (first key, end): enough rows that 128 of them a workgroup fill the chip
@pytest.mark.parametrize("case", [
    (1, 4201, 0, 8, 1, 128, 64, 8, True, None),
    (1, 2100, 3000, 16, 1, 64, 64, 7, True, None),
    (2, 1500, 900, 12, 2, 128, 64, 13, True, None),
    (1, 4100, 77, 8, 1, 64, 64, 24, True, None),
    (1, 4100, 1000, 8, 1, 128, 64, 61, True, None),
    (3, 700, 5000, 16, 8, 128, 128, 4, True, (1280, 4000)),
    (1, 4200, 100, 8, 1, 128, 64, 16, False, None),
    (1, 4200, 0, 8, 1, 64, 4096, 2, True, None),
    (1, 4200, 4000, 8, 1, 128, 64, 1, True, None),
])
def test_selection_of_many_rows(sp, case):
    B, s, off, Hq, Hkv, D, L, top_k, causal, rng_ = case
    say("select many rows %r" % (case,))
    N = off + s
    begin, end = rng_ or (0, N)
    q, q64 = rows((B, s, Hq, D), "q", top_k)
    k, _ = rows((B, N, Hkv, D), "k", top_k)
    means = sp.slimpipe_attn_block_means(k, 0, N, L)
    index = sp.slimpipe_attn_block_select(q, means, off, begin, end, L, top_k, causal).cpu().numpy()
    assert np.array_equal(index, best_blocks(q64, host_f64(means), off, begin // L, -(-end // L), L, top_k, causal))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("s", [5, 4200])
def test_selection_of_degenerate_scores(sp, s, D):
    """Rows of zeros, tiny, huge, infinite and NaN rows; means that are all equal, all zero, tiny, and nearly equal: both kernels, exactly."""
    import torch
    Hq, L, top_k, nb = 8, 64, 5, 150
    off = nb * L
    say("select degenerate s=%d D=%d" % (s, D))
    q, _ = rows((1, s, Hq, D), "q")
    r = torch.arange(s, device="cuda")
    q[:, r % 5 == 1] = 0.0
    q[:, r % 5 == 2] *= 2.0 ** -60
    q[:, r % 5 == 3] *= 2.0 ** -120
    q[0, 4::50, 1] *= 2.0 ** 100
    q[0, 4::50, 2, 3] = float("inf")
    q[0, 4::50, 3, 3] = float("nan")
    q64 = host_f64(q)
    base, _ = rows((nb + 100, 1, 1, D), "k")
    base = base.float()[None, None, :, 0, 0]
    cases = [base, torch.zeros_like(base), torch.ones_like(base), base * 2.0 ** -110, base * 2.0 ** -60, 1.0 + base * 2.0 ** -22]
    half = base.clone()
    half[:, :, ::2] = 0.0
    bad = base.clone()
    bad[0, 0, 7, 1] = float("nan")
    bad[0, 0, 9, 2] = float("inf")
    bad[0, 0, 11, 2] = -float("inf")
    for m in cases + [half, bad]:
        m = m.contiguous()
        got = sp.slimpipe_attn_block_select(q, m, off, 0, nb * L + s, L, top_k).cpu().numpy()
        with np.errstate(invalid="ignore", over="ignore"):
            scores_q = q64
            want = best_blocks(scores_q, host_f64(m), off, 0, -(-(nb * L + s) // L), L, top_k, True)
        # (numpy's order of additions moves a score by D 2^-53 of its terms: where two differ by less, either may come first)
        differ = (got != want).any(-1)
        for b, h, row in zip(*np.nonzero(differ)):
            a, c = set(got[b, h, row].tolist()) - set(want[b, h, row].tolist()), set(want[b, h, row].tolist()) - set(got[b, h, row].tolist())
            x = q64[b, row, h]
            for i in a:
                for j in c:
                    mi, mj = host_f64(m)[0, 0, i], host_f64(m)[0, 0, j]
                    assert abs(math.fsum(x * mi) - math.fsum(x * mj)) <= 2.0 ** -45 * (np.abs(x * mi).sum() + np.abs(x * mj).sum()), (h, row, i, j)
                    assert i < j or math.fsum(x * mi) != math.fsum(x * mj), (h, row, i, j)


def test_lists_of_many_blocks(sp):
    """As many blocks as fit the lists of one launch, more than one window of the lists (1024) and than the lengths that pass through LDS (8192): forward and
    backward."""
    import torch
    B, Hkv, D, L, top_k = 1, 1, 64, 64, 8
    for blocks, s, Hq in ((900, 150, 2), (1500, 150, 2), (8300, 150, 2), (4200, 1024, 4)):      # (the last: with a launch for the chunks' starts)
        N = blocks * L - 17
        off = N - s
        say("many blocks %d" % blocks)
        rng = np.random.default_rng(blocks)
        used = np.unique(np.concatenate([[0, 1023, 1024, blocks - 1, blocks - 2, blocks - 3], rng.integers(0, blocks, 6)]))
        used = used[used < blocks]
        index = np.full((B, Hq, s, top_k), -1, dtype=np.int32)
        for at in np.ndindex(B, Hq, s):
            index[at] = rng.permutation(used)[:top_k]
        pos = np.concatenate([np.arange(j * L, min(N, (j + 1) * L)) for j in used])
        q, q64 = rows((B, s, Hq, D), "q")
        do, do64 = rows((B, s, Hq, D), "do")
        k, v = torch.full((2, B, N, Hkv, D), float("nan"), device="cuda", dtype=torch.bfloat16)
        kk, k64 = rows((B, len(pos), Hkv, D), "k")
        vv, v64 = rows((B, len(pos), Hkv, D), "v")
        at = torch.from_numpy(pos).cuda()
        k[:, at], v[:, at] = kk, vv
        see = (index[..., None] == pos // L).any(-2) & (pos <= (off + np.arange(s))[:, None])
        nan = ~see.any((1, 2))                              # keys that no row sees stay NaN
        k[:, at[torch.from_numpy(nan[0]).cuda()]] = float("nan")
        v[:, at[torch.from_numpy(nan[0]).cuda()]] = float("nan")
        r = bu.Reference(q64, k64, v64, see, 1 / math.sqrt(D), parts_16=True)
        idx = torch.from_numpy(index).cuda()
        out, lse = sp.slimpipe_attn_block_fwd(q, k, v, idx, off, 0, N, L)
        bu.check("out", host_f64(out), r.out, r.out_tol)
        bu.check("lse", host_f64(lse), r.lse, r.lse_tol)
        dk, dv = torch.full((2, B, N, Hkv, D), 5.0, device="cuda")
        dq = sp.slimpipe_attn_block_bwd(q, k, v, idx, out, do, lse, off, 0, N, L, dk, dv, dkv_accumulate=False)
        want = r.backward(host_f64(out), do64, host_f64(lse), True)
        bu.check("dq", host_f64(dq), *want[0])
        bu.check("dk", host_f64(dk[:, at]), *want[1])
        bu.check("dv", host_f64(dv[:, at]), *want[2])
        rest = torch.ones(N, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert (dk[:, rest] == 0).all() and (dv[:, rest] == 0).all()


# rows, offset, heads, kv heads, head_dim, block, top_k, causal, (kv_begin, kv_end): 256 keys a dk/dv workgroup, and lists of several parts
@pytest.mark.parametrize("case", [
    (900, 1100, 4, 1, 64, 256, 3, True, None),
    (900, 1100, 4, 1, 128, 512, 2, True, None),
    (700, 1300, 6, 2, 128, 1024, 2, True, (130, 1999)),
    (800, 1000, 4, 1, 64, 704, 2, True, (700, 1800)),
    (800, 700, 4, 1, 128, 448, 2, False, None),
    (500, 1548, 3, 3, 128, 2048, 1, True, None),
    (600, 900, 4, 2, 64, 576, 3, True, (577, 1500)),
    (820, 700, 4, 1, 128, 320, 2, True, None),
])
def test_backward_of_long_blocks(sp, case):
    import torch
    s, off, Hq, Hkv, D, L, top_k, causal, rng_ = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("long blocks %r" % (case,))
    q, q64 = rows((1, s, Hq, D), "q", L)
    do, do64 = rows((1, s, Hq, D), "do", L)
    k, k64 = rows((1, N, Hkv, D), "k", L)
    v, v64 = rows((1, N, Hkv, D), "v", L)
    rng = np.random.default_rng(L)
    blocks = -(-N // L)
    index = np.stack([rng.permutation(blocks)[:top_k] if top_k <= blocks else np.resize(np.arange(blocks), top_k) for _ in range(Hq * s)])
    index[rng.random(len(index)) < 0.8, 0] = begin // L       # most rows on one block (and then maybe twice)
    index = index.reshape(1, Hq, s, top_k).astype(np.int32)
    r = bu.Reference(q64, k64, v64, bu.visible(index, off, begin, end, L, causal, N), 1 / math.sqrt(D), parts_16=True)
    idx = torch.from_numpy(index).cuda()
    out, lse = sp.slimpipe_attn_block_fwd(q, k, v, idx, off, begin, end, L, causal)
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)
    dk, dv = torch.full((2, 1, N, Hkv, D), 5.0, device="cuda")
    dq = sp.slimpipe_attn_block_bwd(q, k, v, idx, out, do, lse, off, begin, end, L, dk, dv, causal, dkv_accumulate=False)
    want = r.backward(host_f64(out), do64, host_f64(lse), True)
    bu.check("dq", host_f64(dq), *want[0])
    for name, x, (w, tol) in (("dk", dk, want[1]), ("dv", dv, want[2])):
        got = host_f64(x)
        assert (got[:, :begin] == 5.0).all() and (got[:, end:] == 5.0).all()
        bu.check(name, got[:, begin:end], w[:, begin:end], tol[:, begin:end])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("begin", [371, 510, 253])
def test_backward_of_chunks_behind_an_odd_first_key(sp, D, begin):
    """Lists in several parts on either side of a chunk's end, in a range that starts at any key: each key's sums go to its own chunk, and what
    lies behind the chunks stays as it was."""
    import torch
    s, off, Hq, L, C = 520, 400, 8, 64, 256
    N = off + s
    say("chunked reduce D=%d begin=%d" % (D, begin))
    q, q64 = rows((1, s, Hq, D), "q")
    do, do64 = rows((1, s, Hq, D), "do")
    k, k64 = rows((1, N, 1, D), "k")
    v, v64 = rows((1, N, 1, D), "v")
    index = np.tile(np.array([3, 4, 7, 8, 11, 12], dtype=np.int32), (1, Hq, s, 1))
    idx = torch.from_numpy(index).cuda()
    kc, vc = ([torch.nn.functional.pad(x[:, i:i + C], (0, 0, 0, 0, 0, max(0, i + C - N))).contiguous() for i in range(0, N, C)] for x in (k, v))
    out, lse = sp.slimpipe_attn_block_fwd(q, kc, vc, idx, off, begin, N, L)
    r = bu.Reference(q64, k64, v64, bu.visible(index, off, begin, N, L, True, N), 1 / math.sqrt(D), parts_16=True)
    bu.check("out", host_f64(out), r.out, r.out_tol)
    # every chunk's accumulator with a margin of 64 rows on either side
    room = [torch.full((1, C + 128, 1, D), 2.0, device="cuda") for _ in range(2 * len(kc))]
    acc = [x[:, 64:64 + C] for x in room]
    dkc, dvc = acc[:len(kc)], acc[len(kc):]
    sp.slimpipe_attn_block_bwd(q, kc, vc, idx, out, do, lse, off, begin, N, L, dkc, dvc)
    assert all((x[:, :64] == 2.0).all() and (x[:, 64 + C:] == 2.0).all() for x in room)
    want = r.backward(host_f64(out), do64, host_f64(lse), True)
    for name, chunks, (w, tol) in (("dk", dkc, want[1]), ("dv", dvc, want[2])):
        got = host_f64(torch.cat(chunks, 1))
        assert (got[:, :begin] == 2.0).all() and (got[:, N:] == 2.0).all()
        bu.check(name, got[:, begin:N] - 2.0, w[:, begin:], tol[:, begin:] + 2.0 ** -22 * (2.0 + np.abs(w[:, begin:])))


@pytest.mark.parametrize("s", [3, 300])
def test_nan_is_not_dropped(sp, s):
    """A NaN among what a row sees makes its out and lse NaN, in either form of both attentions, and leaves rows alone that do not see it."""
    import torch
    Hq, Hkv, D, L, top_k, off = 4, 2, 64, 64, 3, 640
    N = off + s
    q, _ = rows((1, s, Hq, D), "q")
    k, _ = rows((1, N, Hkv, D), "k")
    v, _ = rows((1, N, Hkv, D), "v")
    index = torch.tensor([0, 2, 5], device="cuda", dtype=torch.int32).expand(1, Hq, s, top_k).contiguous()
    index[:, :, 1::2, 1] = 3
    clean = sp.slimpipe_attn_block_fwd(q, k, v, index, off, 0, N, L)
    q2, k2 = q.clone(), k.clone()
    q2[0, 0, 1, 7] = float("nan")                             # one row
    k2[0, 2 * L + 5, 1, 3] = float("nan")                     # block 2 of kv head 1: even rows of heads 2, 3
    hit = torch.zeros((1, Hq, s), dtype=torch.bool, device="cuda")
    hit[0, 1, 0] = True
    hit[0, 2:, ::2] = True
    out, lse = sp.slimpipe_attn_block_fwd(q2, k2, v, index, off, 0, N, L)
    assert torch.equal(torch.isnan(lse), hit) and torch.equal(lse[~hit], clean[1][~hit])
    rows_hit = hit.permute(0, 2, 1)
    assert torch.isnan(out[rows_hit]).all() and torch.equal(out[~rows_hit], clean[0][~rows_hit])
    # the cache: a group with an infinity reads as NaN
    cache = sp.KvCache4.empty(1, N, Hkv, D)
    k2 = k.clone()
    sp.slimpipe_attn_kv4_store(k2, v, cache, 0)
    clean = sp.slimpipe_attn_fwd_kv4(q, cache, off, 0, off)
    k2[0, 100, 1, 3] = float("inf")
    sp.slimpipe_attn_kv4_store(k2[:, 100:101], v[:, 100:101], cache, 100)
    out, lse = sp.slimpipe_attn_fwd_kv4(q, cache, off, 0, off)
    assert torch.isnan(lse[:, 2:]).all() and torch.isnan(out[:, :, 2:]).all()
    assert torch.equal(lse[:, :2], clean[1][:, :2]) and torch.equal(out[:, :, :2], clean[0][:, :, :2])
    # a value: the columns of its group
    v2 = v.clone()
    v2[0, 33, 0, 40] = float("nan")
    sp.slimpipe_attn_kv4_store(k, v2, cache, 0)
    out, lse = sp.slimpipe_attn_fwd_kv4(q, cache, off, 0, off)
    assert torch.equal(lse, clean[1])
    assert torch.isnan(out[:, :, :2, 32:]).all() and torch.equal(out[..., :32], clean[0][..., :32]) and torch.equal(out[:, :, 2:], clean[0][:, :, 2:])


def test_offsets_past_32_bits(sp):
    """The last keys of caches of more than 2^32 elements: as the same keys in a small one."""
    import torch
    B, s, Hq, Hkv, D, L, n = 1, 200, 8, 8, 128, 64, 640
    N = (1 << 32) // (Hkv * D) + n
    off = N - s
    assert N % L == 0 and (N - n) * Hkv * D == 1 << 32
    q, _ = rows((B, s, Hq, D), "q")
    do, _ = rows((B, s, Hq, D), "do")
    k, _ = rows((B, n, Hkv, D), "k")
    v, _ = rows((B, n, Hkv, D), "v")
    small = torch.from_numpy(np.random.default_rng(1).integers(0, n // L, (B, Hq, s, 3), dtype=np.int32)).cuda()
    first = (N - n) // L
    far = [torch.empty((B, N, Hkv, D), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    for x, y in zip(far, (k, v)):
        x[:, N - n:] = y
    m0 = sp.slimpipe_attn_block_means(k, 0, n, L)
    m1 = sp.slimpipe_attn_block_means(far[0], N - n, N, L, means=torch.empty((B, Hkv, N // L, D), device="cuda"))
    assert torch.equal(m0, m1[:, :, first:])
    assert torch.equal(sp.slimpipe_attn_block_select(q, m0, n - s, 0, n, L, 4) + first, sp.slimpipe_attn_block_select(q, m1, off, N - n, N, L, 4))
    for rows_ in (slice(None), slice(0, 2)):
        a = sp.slimpipe_attn_block_fwd(q[:, rows_], k, v, small[:, :, rows_].contiguous(), n - s, 0, n, L)
        b = sp.slimpipe_attn_block_fwd(q[:, rows_], *far, small[:, :, rows_].contiguous() + first, off, N - n, N, L)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out, lse = sp.slimpipe_attn_block_fwd(q, k, v, small, n - s, 0, n, L)
    dk, dv = torch.zeros((2, B, n, Hkv, D), device="cuda")
    dq = sp.slimpipe_attn_block_bwd(q, k, v, small, out, do, lse, n - s, 0, n, L, dk, dv)
    grads = [torch.empty((B, N, Hkv, D), device="cuda") for _ in range(2)]
    dq2 = sp.slimpipe_attn_block_bwd(q, *far, small + first, out, do, lse, off, N - n, N, L, *grads, dkv_accumulate=False)
    assert torch.equal(dq, dq2) and torch.equal(dk, grads[0][:, N - n:]) and torch.equal(dv, grads[1][:, N - n:])
    del grads, far
    caches = [sp.KvCache4(*(torch.empty((B, rows_, Hkv, w), device="cuda", dtype=torch.uint8) for w in (D // 2, D // 32, D // 2, D // 32))) for rows_ in (n, N)]
    for cache, at in zip(caches, (0, N - n)):
        sp.slimpipe_attn_kv4_store(k, v, cache, at)
    assert all(torch.equal(x, y[:, N - n:]) for x, y in zip(*caches))
    assert all(torch.equal(x, y) for x, y in zip(sp.slimpipe_attn_kv4_load(caches[0], 0, n), sp.slimpipe_attn_kv4_load(caches[1], N - n, N)))
    for rows_ in (slice(None), slice(0, 2)):
        a = sp.slimpipe_attn_fwd_kv4(q[:, rows_], caches[0], n - s, 0, n)
        b = sp.slimpipe_attn_fwd_kv4(q[:, rows_], caches[1], off, N - n, N)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # batches far apart: the second one's rows lie past 2^32 elements
    wide = sp.KvCache4(*(torch.empty_strided((2, n, Hkv, w), ((N + 32) * Hkv * w, Hkv * w, w, 1), device="cuda", dtype=torch.uint8) for w in (D // 2, D // 32, D // 2, D // 32)))
    both = torch.cat([k.flip(1), k]), torch.cat([v.flip(1), v])
    sp.slimpipe_attn_kv4_store(*both, wide, 0)
    got, want = sp.slimpipe_attn_fwd_kv4(torch.cat([q, q]), wide, n - s, 0, n), sp.slimpipe_attn_fwd_kv4(q, caches[0], n - s, 0, n)
    assert torch.equal(got[0][1:], want[0]) and torch.equal(got[1][1:], want[1])


def test_two_streams_and_two_graphs(sp):
    """Calls on two streams at once, each with its own workspace; two graphs captured over one workspace and replayed in turn."""
    import torch
    Hq, Hkv, D, L, top_k, s, off = 8, 2, 128, 64, 4, 700, 500
    N = off + s
    sets = []
    for i in range(2):
        t = {n: rows((1, r, h, D), n, 50 + i)[0] for n, r, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv), ("do", s, Hq))}
        t["index"] = torch.from_numpy(np.random.default_rng(i).integers(0, N // L, (1, Hq, s, top_k), dtype=np.int32)).cuda()
        t["cache"] = sp.KvCache4.empty(1, N, Hkv, D)
        sp.slimpipe_attn_kv4_store(t["k"], t["v"], t["cache"], 0)
        sets.append(t)
    size = sp.slimpipe_attn_block_workspace_bytes(sets[0]["q"], sets[0]["k"], sets[0]["index"], off, 0, N, L, True, True)
    size4 = sp.slimpipe_attn_kv4_workspace_bytes(sets[0]["q"], sets[0]["cache"], off, 0, N)
    ws = [torch.empty(max(size, size4), device="cuda", dtype=torch.uint8) for _ in range(2)]

    def step(t, w):
        o, l = sp.slimpipe_attn_block_fwd(t["q"], t["k"], t["v"], t["index"], off, 0, N, L, workspace=w)
        dk, dv = torch.zeros((2, 1, N, Hkv, D), device="cuda")
        dq = sp.slimpipe_attn_block_bwd(t["q"], t["k"], t["v"], t["index"], o, t["do"], l, off, 0, N, L, dk, dv, workspace=w)
        o4, l4 = sp.slimpipe_attn_fwd_kv4(t["q"], t["cache"], off, 0, N, workspace=w)
        chosen = sp.slimpipe_attn_block_select(t["q"], sp.slimpipe_attn_block_means(t["k"], 0, N, L), off, 0, N, L, top_k)
        return o, l, dq, dk, dv, o4, l4, chosen
    want = [step(t, w) for t, w in zip(sets, ws)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        got = []
        for st, t, w in zip(streams, sets, ws):
            with torch.cuda.stream(st):
                got.append(step(t, w))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, e in zip(got, want) for x, y in zip(g, e))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g, t in zip(graphs, sets):
        with torch.cuda.graph(g):
            outs.append(step(t, ws[0]))
    for i in (0, 1, 1, 0, 1, 0):
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[i], want[i])), i
        step(sets[1 - i], ws[0])
        torch.cuda.synchronize()


def test_training_step_over_slices(sp):
    """A sequence in three slices over a chunked cache, as a pipeline stage trains on it: means as the cache grows, choice, forward; then the slices
    backwards, dk and dv added up over them and rounded at the end.  Against the sum of the slices' 64-bit gradients."""
    import torch
    B, Hq, Hkv, D, L, top_k, s, n = 2, 4, 2, 64, 64, 3, 256, 3
    N = s * n
    q, q64 = rows((B, N, Hq, D), "q", 3)
    do, do64 = rows((B, N, Hq, D), "do", 3)
    k, k64 = rows((B, N, Hkv, D), "k", 3)
    v, v64 = rows((B, N, Hkv, D), "v", 3)
    kc, vc = ([x[:, i * s:(i + 1) * s].contiguous() for i in range(n)] for x in (k, v))
    means = torch.zeros((B, Hkv, N // L, D), device="cuda")
    saved = []
    for i in range(n):
        qi, end = q[:, i * s:(i + 1) * s], (i + 1) * s
        sp.slimpipe_attn_block_means(kc, i * s, end, L, means=means)
        index = sp.slimpipe_attn_block_select(qi, means, i * s, 0, end, L, top_k)
        assert np.array_equal(index.cpu().numpy(), bu.select(host_f64(qi), host_f64(means), i * s, 0, end, L, top_k, True))
        saved.append((qi, index, *sp.slimpipe_attn_block_fwd(qi, kc, vc, index, i * s, 0, end, L)))
    dkc, dvc = ([torch.zeros(x.shape, device="cuda") for x in kc] for _ in range(2))
    want = [np.zeros((B, N, Hkv, D)) for _ in range(4)]
    for i in reversed(range(n)):
        qi, index, out, lse = saved[i]
        end = (i + 1) * s
        r = bu.Reference(host_f64(qi), k64, v64, bu.visible(index.cpu().numpy(), i * s, 0, end, L, True, N), 1 / math.sqrt(D), parts_16=True)
        bu.check("out %d" % i, host_f64(out), r.out, r.out_tol)
        bu.check("lse %d" % i, host_f64(lse), r.lse, r.lse_tol)
        dq = sp.slimpipe_attn_block_bwd(qi, kc, vc, index, out, do[:, i * s:end], lse, i * s, 0, end, L, dkc, dvc)
        g = r.backward(host_f64(out), do64[:, i * s:end], host_f64(lse), True)
        bu.check("dq %d" % i, host_f64(dq), *g[0])
        for at, x in enumerate((*g[1], *g[2])):
            want[at] += x
    for name, acc, w, tol in (("dk", dkc, want[0], want[1]), ("dv", dvc, want[2], want[3])):
        # one float32 addition a slice, one rounding to bf16
        got = torch.cat([sp.slimpipe_attn_finalize_bf16(x) for x in acc], 1)
        bu.check(name, host_f64(got), w, tol * (1 + 2.0 ** -7) + (bu.HALF_BF16 + n * 2.0 ** -23) * np.abs(w))


@pytest.mark.parametrize("power", [100, -60])
def test_values_of_any_magnitude(sp, power):
    """Values and upstream gradients far from 1: 16-bit partial results keep their bits.  An infinite value leaves the other columns alone."""
    import torch
    s, off, Hq, Hkv, D, L, top_k = 300, 468, 4, 2, 128, 64, 4
    N = off + s
    say("magnitude 2^%d" % power)
    q, q64 = rows((1, s, Hq, D), "q")
    k, k64 = rows((1, N, Hkv, D), "k")
    v, v64 = rows((1, N, Hkv, D), "v")
    do, do64 = rows((1, s, Hq, D), "do")
    v, v64 = v * 2.0 ** power, v64 * 2.0 ** power
    do, do64 = do * 2.0 ** -power, do64 * 2.0 ** -power
    index = np.random.default_rng(9).integers(0, N // L, (1, Hq, s, top_k), dtype=np.int32)
    idx = torch.from_numpy(index).cuda()
    r = bu.Reference(q64, k64, v64, bu.visible(index, off, 0, N, L, True, N), 1 / math.sqrt(D), parts_16=True)
    out, lse = sp.slimpipe_attn_block_fwd(q, k, v, idx, off, 0, N, L)
    bu.check("out", host_f64(out), r.out, r.out_tol)
    dk, dv = torch.zeros((2,) + k.shape, device="cuda")
    # (the gradients: with v and d_out both scaled dP keeps its size; then d_out alone, and dq is as small or large as it)
    for scaled, scaled64 in ((do, do64), (do * 2.0 ** -20, do64 * 2.0 ** -20)):
        dq = sp.slimpipe_attn_block_bwd(q, k, v, idx, out, scaled, lse, off, 0, N, L, dk, dv)
        want = r.backward(host_f64(out), scaled64, host_f64(lse), True)
        bu.check("dq", host_f64(dq), *want[0])
    v[0, 5, :, 40] = float("inf")
    index[..., 0] = 0                                         # every row sees key 5
    idx = torch.from_numpy(index).cuda()
    r = bu.Reference(q64, k64, v64, bu.visible(index, off, 0, N, L, True, N), 1 / math.sqrt(D), parts_16=True)
    out, _ = sp.slimpipe_attn_block_fwd(q, k, v, idx, off, 0, N, L)
    got, rest = host_f64(out), np.arange(D) != 40
    assert np.isinf(got[..., 40]).all()
    bu.check("the other columns", got[..., rest], r.out[..., rest], r.out_tol[..., rest])


@pytest.mark.parametrize("s,L,D", [(60, 64, 64), (700, 64, 64), (700, 256, 128)])
def test_gradients_over_out_and_lse(sp, s, L, D):
    """dq in place of out and dv over lse: both are read before any gradient is written."""
    import torch
    Hq, Hkv, top_k, off = 4, 1, 4, 900
    N = off + s
    q, _ = rows((1, s, Hq, D), "q")
    do, _ = rows((1, s, Hq, D), "do")
    k, _ = rows((1, N, Hkv, D), "k")
    v, _ = rows((1, N, Hkv, D), "v")
    index = torch.from_numpy(np.random.default_rng(s).integers(0, -(-N // L), (1, Hq, s, top_k), dtype=np.int32)).cuda()
    out, lse = sp.slimpipe_attn_block_fwd(q, k, v, index, off, 0, N, L)
    dk, dv = torch.zeros((2,) + k.shape, device="cuda")
    dq = sp.slimpipe_attn_block_bwd(q, k, v, index, out, do, lse, off, 0, N, L, dk, dv)
    dv2 = torch.zeros_like(dv)
    lse2 = dv2.view(-1)[:lse.numel()].view(lse.shape)
    lse2.copy_(lse)
    dk2, out2 = torch.zeros_like(dk), out.clone()
    sp.slimpipe_attn_block_bwd(q, k, v, index, out2, do, lse2, off, 0, N, L, dk2, dv2, dq=out2, dkv_accumulate=False)
    assert torch.equal(out2, dq) and torch.equal(dk2, dk) and torch.equal(dv2, dv)


def test_calls_from_two_threads(sp):
    """Two host threads, a stream and a workspace each: the results of each call on its own."""
    import threading
    import torch
    s, off, Hq, Hkv, D, L, top_k = 300, 700, 8, 2, 128, 64, 5
    N = off + s
    sets = []
    for i in range(2):
        t = [rows((1, n, h, D), tag, 70 + i)[0] for tag, n, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv), ("do", s, Hq))]
        cache = sp.KvCache4.empty(1, N, Hkv, D)
        sp.slimpipe_attn_kv4_store(t[1], t[2], cache, 0)
        sets.append(t + [cache])

    def work(q, k, v, do, cache):
        means = sp.slimpipe_attn_block_means(k, 0, N, L)
        index = sp.slimpipe_attn_block_select(q, means, off, 0, N, L, top_k)
        out, lse = sp.slimpipe_attn_block_fwd(q, k, v, index, off, 0, N, L)
        dk, dv = torch.zeros((2,) + k.shape, device="cuda")
        dq = sp.slimpipe_attn_block_bwd(q, k, v, index, out, do, lse, off, 0, N, L, dk, dv)
        return index, out, lse, dq, dk, dv, *sp.slimpipe_attn_fwd_kv4(q, cache, off, 0, N)
    want = [work(*t) for t in sets]
    torch.cuda.synchronize()
    bad = []

    def run(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = work(*sets[i])
                stream.synchronize()
                if not all(torch.equal(x, y) for x, y in zip(got, want[i])):
                    bad.append(i)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
