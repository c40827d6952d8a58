"""Sparse attention over selected key blocks on the GPU, against plain 64-bit definitions (tests/block_util.py)."""
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


def tensors(B, s, N, Hq, Hkv, D, salt=0):
    bits = {t: normal_bf16((B, n, H, D), 31, t, salt) for t, n, H in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv), ("do", s, Hq))}
    return {t: dev_bf16(x) for t, x in bits.items()}, {t: bf16_bits_to_f64(x) for t, x in bits.items()}


def random_index(rng, B, Hq, s, top_k, blocks, wild):
    """Any order, gaps, -1; `wild`: also repeated and impossible entries."""
    index = np.full((B, Hq, s, top_k), -1, dtype=np.int32)
    for at in np.ndindex(B, Hq, s):
        n = int(rng.integers(0, min(top_k, blocks) + 1))
        index[at][rng.permutation(top_k)[:n]] = rng.permutation(blocks)[:n]
    if wild:
        hit = rng.random(index.shape) < 0.15
        index[hit] = rng.choice([-2, blocks, blocks + 7, 2 ** 31 - 1, -2 ** 31, 0, blocks - 1], size=int(hit.sum()))
    return index


# batch, rows, offset, heads, kv heads, head_dim, block, top_k, causal, (kv_begin, kv_end) or None
SHAPES = [
    (1, 1, 0, 1, 1, 128, 64, 1, True, None),            # one token on itself
    (2, 1, 700, 8, 1, 128, 64, 5, True, None),          # tokens: a workgroup a (row, slot)
    (1, 3, 1021, 4, 4, 64, 128, 64, True, None),        # more slots than blocks
    (1, 257, 0, 8, 1, 128, 64, 3, True, None),          # first slice, odd length
    (2, 200, 811, 6, 2, 64, 64, 7, True, None),
    (1, 300, 500, 4, 1, 128, 192, 4, True, None),       # a block length that is no power of two
    (1, 600, 900, 2, 2, 128, 256, 2, True, None),       # several 512-row chunks of the lists
    (1, 330, 700, 3, 1, 64, 320, 3, False, None),       # not causal
    (1, 260, 500, 4, 2, 128, 64, 6, True, (100, 650)),  # a part of the keys: rows without any, first block cut
    (1, 260, 500, 4, 2, 64, 128, 3, True, (700, 760)),
    (1, 300, 100, 2, 1, 128, 64, 4, True, (390, 400)),  # a range that few rows see
    (1, 300, 100, 2, 1, 128, 64, 4, True, (250, 250)),  # an empty range
]


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("case", SHAPES)
def test_forward(sp, case, wild):
    import torch
    B, s, off, Hq, Hkv, D, L, top_k, causal, rng_ = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("block forward %r wild=%s" % (case, wild))
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=top_k)
    index = random_index(np.random.default_rng(s + D), B, Hq, s, top_k, -(-N // L), wild)
    see = bu.visible(index, off, begin, end, L, causal, N)
    for dtype in (sp.BF16, sp.F32):
        r = bu.Reference(ref["q"], ref["k"], ref["v"], see, 1 / math.sqrt(D), dtype == sp.BF16, dtype == sp.BF16)
        out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], torch.from_numpy(index).cuda(), off, begin, end, L, causal, out_dtype=dtype)
        torch.cuda.synchronize()
        bu.check("out", host_f64(out), r.out, r.out_tol)
        bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


@pytest.mark.parametrize("case", [
    (2, 1, 700, 8, 1, 128, 64, 5, True, None),
    (1, 70, 0, 4, 4, 64, 64, 2, True, None),
    (1, 100, 1500, 6, 2, 64, 128, 16, True, None),
    (2, 37, 333, 3, 1, 128, 192, 1, True, None),
    (1, 40, 600, 2, 2, 128, 64, 4, False, None),
    (1, 90, 500, 4, 1, 128, 64, 3, True, (128, 530)),
    (1, 20, 100, 2, 1, 64, 64, 3, True, (64, 64)),
    (1, 5, 40000, 4, 1, 64, 64, 64, True, None),        # more blocks than one chunk of the selection
    (1, 3, 60000, 4, 1, 128, 64, 24, True, None),       # scores of more tiles a wave than two, all of them kept
    (1, 2, 140000, 8, 1, 64, 64, 8, True, None),        # and more than are kept
])
def test_means_and_selection(sp, case):
    import torch
    B, s, off, Hq, Hkv, D, L, top_k, causal, rng_ = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("block select %r" % (case,))
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=7)
    means = sp.slimpipe_attn_block_means(dev["k"], 0, N, L)
    want = bu.means(ref["k"], 0, N, L)
    got = host_f64(means)
    for j, m in want.items():
        assert np.abs(got[:, :, j] - m).max() <= 2.0 ** -24 * np.abs(m).max() * 1.01, j
    index = sp.slimpipe_attn_block_select(dev["q"], means, off, begin, end, L, top_k, causal)
    torch.cuda.synchronize()
    assert np.array_equal(index.cpu().numpy(), bu.select(ref["q"], got, off, begin, end, L, top_k, causal))


def test_selection_ties_and_nan(sp):
    """Equal means: the lowest indices.  A difference that 32 bits do not show decides.  NaN comes last."""
    import torch
    D, L, nb = 64, 64, 700
    q = torch.ones((1, 2, 1, D), device="cuda").bfloat16()
    means = torch.zeros((1, 1, nb, D), device="cuda")
    off = nb * L - 2
    index = sp.slimpipe_attn_block_select(q, means, off, 0, nb * L, L, 9)
    assert index[0, 0].tolist() == [[0, 1, 2, 3, 4, 5, 6, 7, nb - 1]] * 2
    means[:, :, :, 0] = 1.0
    means[0, 0, 650, 1] = 2.0 ** -40                       # 1 + 2^-40 rounds to 1 in 32 bits
    means[0, 0, 20, 1] = 2.0 ** -41
    means[0, 0, 3] = float("nan")
    index = sp.slimpipe_attn_block_select(q, means, off, 0, nb * L, L, 5)
    assert index[0, 0].tolist() == [[0, 1, 20, 650, nb - 1]] * 2
    index = sp.slimpipe_attn_block_select(q, means, off, 0, nb * L, L, 4, causal=False)
    assert index[0, 0].tolist() == [[0, 1, 20, 650]] * 2
    means[:] = float("nan")
    index = sp.slimpipe_attn_block_select(q, means, off, 0, nb * L, L, 3)
    assert index[0, 0].tolist() == [[0, 1, nb - 1]] * 2


def test_means_grow_with_the_cache(sp):
    """Slice by slice the same means as at once, other blocks untouched, from a chunk list too."""
    import torch
    dev, _ = tensors(2, 8, 1100, 2, 2, 64)
    whole = sp.slimpipe_attn_block_means(dev["k"], 0, 1100, 128)
    grown = torch.full_like(whole, 7.0)
    pos = 0
    for n in (300, 1, 211, 588):
        sp.slimpipe_attn_block_means(dev["k"], pos // 128 * 128, pos + n, 128, means=grown)
        pos += n
        assert (grown[:, :, -(-pos // 128):] == 7.0).all()
    assert torch.equal(whole, grown)
    chunks = [torch.zeros_like(dev["k"][:, :512]) for _ in range(3)]
    for i, c in enumerate(chunks):
        part = dev["k"][:, i * 512:(i + 1) * 512]
        c[:, :part.shape[1]] = part
    from_list = sp.slimpipe_attn_block_means(chunks, 0, 1100, 128)
    assert torch.equal(from_list[:, :, :9], whole) and (from_list[:, :, 9:] == 0).all()


def test_all_blocks_chosen_is_dense(sp):
    """With every block of the prefix chosen the result is the dense call's, to the rounding of both."""
    import torch
    B, s, off, Hq, Hkv, D, L = 1, 384, 640, 8, 2, 128, 64
    dev, ref = tensors(B, s, off + s, Hq, Hkv, D, salt=3)
    index = torch.arange(16, device="cuda", dtype=torch.int32).expand(B, Hq, s, 16).contiguous()
    out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], index, off, 0, off + s, L)
    dense, dense_lse = sp.slimpipe_attn_fwd(dev["q"], dev["k"], dev["v"], off, 0, off + s)
    see = np.broadcast_to(np.arange(off + s) <= (off + np.arange(s))[:, None], (B, Hq, s, off + s))
    r = bu.Reference(ref["q"], ref["k"], ref["v"], see, 1 / math.sqrt(D), parts_16=True)
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("out against dense", host_f64(out), host_f64(dense), 2 * r.out_tol)
    bu.check("lse against dense", host_f64(lse), host_f64(dense_lse), 2 * r.lse_tol)


def test_forward_layouts_chunks_and_unseen_keys(sp):
    """Strided heads, a chunk list, and NaN in every key that no row sees: the same bits as plain contiguous inputs."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = 2, 150, 618, 6, 2, 64, 128, 3
    N = off + s
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=5)
    index = random_index(np.random.default_rng(0), B, Hq, s, top_k, -(-N // L), True)
    idx = torch.from_numpy(index).cuda()
    out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], idx, off, 0, N, L)
    see = bu.visible(index, off, 0, N, L, True, N).reshape(B, Hkv, Hq // Hkv, s, N).any((2, 3)).transpose(0, 2, 1)      # [B, N, Hkv]
    qkv = torch.zeros((B, s, 3 * Hq, D), device="cuda", dtype=torch.bfloat16)
    q2 = qkv[:, :, Hq:2 * Hq]
    q2.copy_(dev["q"])
    k2, v2 = torch.full((2, B, N + 200, Hkv, D), float("nan"), device="cuda", dtype=torch.bfloat16)
    mask = torch.from_numpy(np.ascontiguousarray(see)).cuda()[..., None]
    nan = torch.tensor(float("nan"), device="cuda", dtype=torch.bfloat16)
    k2[:, :N], v2[:, :N] = torch.where(mask, dev["k"], nan), torch.where(mask, dev["v"], nan)
    o2, l2 = sp.slimpipe_attn_block_fwd(q2, k2, v2, idx, off, 0, N, L)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    kc = [k2[:, i:i + 256].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for i in range(0, 768, 256)]
    vc = [v2[:, i:i + 256].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for i in range(0, 768, 256)]
    o3, l3 = sp.slimpipe_attn_block_fwd(q2, kc, vc, idx, off, 0, N, L)
    assert torch.equal(out, o3) and torch.equal(lse, l3)


def test_ranges_merge_to_the_whole(sp):
    """(out, lse) over two key ranges, folded by slimpipe_attn_merge, are the call over both."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = 1, 200, 700, 4, 1, 128, 64, 5
    N = off + s
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=9)
    means = sp.slimpipe_attn_block_means(dev["k"], 0, N, L)
    idx = sp.slimpipe_attn_block_select(dev["q"], means, off, 0, N, L, top_k)
    parts = [sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], idx, off, a, b, L, out_dtype=sp.F32) for a, b in ((0, 333), (333, N))]
    out, lse = sp.slimpipe_attn_merge([p[0] for p in parts], [p[1] for p in parts])
    r = bu.Reference(ref["q"], ref["k"], ref["v"], bu.visible(idx.cpu().numpy(), off, 0, N, L, True, N), 1 / math.sqrt(D))
    bu.check("out", host_f64(out), r.out, r.out_tol)
    bu.check("lse", host_f64(lse), r.lse, r.lse_tol)


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("case", SHAPES)
def test_backward(sp, case, wild):
    import torch
    B, s, off, Hq, Hkv, D, L, top_k, causal, rng_ = case
    N = off + s
    begin, end = rng_ or (0, N)
    say("block backward %r wild=%s" % (case, wild))
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=top_k + 100)
    index = random_index(np.random.default_rng(s + D), B, Hq, s, top_k, -(-N // L), wild)
    idx = torch.from_numpy(index).cuda()
    r = bu.Reference(ref["q"], ref["k"], ref["v"], bu.visible(index, off, begin, end, L, causal, N), 1 / math.sqrt(D), parts_16=True)
    out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], idx, off, begin, end, L, causal)
    dk, dv = torch.full((2,) + dev["k"].shape, 3.0, device="cuda")
    dq = sp.slimpipe_attn_block_bwd(dev["q"], dev["k"], dev["v"], idx, out, dev["do"], lse, off, begin, end, L, dk, dv, causal, dkv_accumulate=wild)
    torch.cuda.synchronize()
    want = r.backward(host_f64(out), ref["do"], host_f64(lse), True)
    bu.check("dq", host_f64(dq), *want[0])
    for name, x, (w, tol) in (("dk", dk, want[1]), ("dv", dv, want[2])):
        got = host_f64(x)
        assert (got[:, :begin] == 3.0).all() and (got[:, end:] == 3.0).all(), name      # rows outside the range stay
        if wild:                                                                       # added to what was there: one float32 rounding more
            got, tol = got - 3.0, tol + 2.0 ** -23 * (3.0 + np.abs(w))
        bu.check(name, got[:, begin:end], w[:, begin:end], tol[:, begin:end])


def test_backward_long_lists_layouts_and_repeats(sp):
    """Lists longer than one workgroup's part, from chunk lists, dq in float32 added to what is there; the same bits again, and with NaN in
    the keys that no row sees."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = 1, 1500, 548, 6, 1, 64, 128, 3
    N = off + s
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=8)
    index = random_index(np.random.default_rng(3), B, Hq, s, top_k, 10, False)
    index[..., 0] = 2                                       # 9000 rows on one block
    idx = torch.from_numpy(index).cuda()
    see = bu.visible(index, off, 0, N, L, True, N)
    r = bu.Reference(ref["q"], ref["k"], ref["v"], see, 1 / math.sqrt(D))
    out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], idx, off, 0, N, L)
    want = r.backward(host_f64(out), ref["do"], host_f64(lse), False)
    nan = torch.tensor(float("nan"), device="cuda", dtype=torch.bfloat16)
    mask = torch.from_numpy(np.ascontiguousarray(see.any((1, 2)))).cuda()[:, :, None, None]
    first = None
    for k, v in ((dev["k"], dev["v"]), (dev["k"], dev["v"]), (torch.where(mask, dev["k"], nan), torch.where(mask, dev["v"], nan))):
        kc, vc = ([x[:, i:i + 1024].contiguous() for i in (0, 1024)] for x in (k, v))
        dkc, dvc = ([torch.full(x.shape, 9.0, device="cuda") for x in kc] for _ in range(2))
        dq = torch.ones((B, s, Hq, D), device="cuda")
        sp.slimpipe_attn_block_bwd(dev["q"], kc, vc, idx, out, dev["do"], lse, off, 0, N, L, dkc, dvc, dq=dq, dq_dtype=sp.F32, dq_accumulate=True,
                                   dkv_accumulate=False)
        got = dq, torch.cat(dkc, 1), torch.cat(dvc, 1)
        if first is None:
            first = got
            bu.check("dq", host_f64(dq) - 1.0, want[0][0], want[0][1] + 2.0 ** -23 * (1.0 + np.abs(want[0][0])))
            bu.check("dk", host_f64(got[1]), *want[1])
            bu.check("dv", host_f64(got[2]), *want[2])
        assert all(torch.equal(x, y) for x, y in zip(first, got))


def test_gradients_against_differences(sp):
    """dq, dk, dv against central differences of the 64-bit forward along random directions, as far as the call's roundings allow."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = 1, 48, 160, 4, 2, 64, 64, 2
    N = off + s
    dev, ref = tensors(B, s, N, Hq, Hkv, D, salt=21)
    index = random_index(np.random.default_rng(5), B, Hq, s, top_k, -(-N // L), False)
    idx = torch.from_numpy(index).cuda()
    see = bu.visible(index, off, 0, N, L, True, N)
    scale = 1 / math.sqrt(D)
    out, lse = sp.slimpipe_attn_block_fwd(dev["q"], dev["k"], dev["v"], idx, off, 0, N, L)
    dk, dv = torch.zeros((2,) + dev["k"].shape, device="cuda")
    dq = sp.slimpipe_attn_block_bwd(dev["q"], dev["k"], dev["v"], idx, out, dev["do"], lse, off, 0, N, L, dk, dv, dq_dtype=sp.F32)
    r = bu.Reference(ref["q"], ref["k"], ref["v"], see, scale)
    rng, eps = np.random.default_rng(6), 1e-5
    want = r.backward(host_f64(out), ref["do"], host_f64(lse), False)
    exact = r.backward(r.out, ref["do"], r.lse, False)
    for i, (name, got) in enumerate((("q", dq), ("k", dk), ("v", dv))):
        step = rng.standard_normal(ref[name].shape)
        f = [(bu.Reference(*(ref[t] + (sign * eps * step if t == name else 0.0) for t in "qkv"), see, scale).out * ref["do"]).sum() for sign in (1, -1)]
        slope = (f[0] - f[1]) / (2 * eps)
        assert abs((exact[i][0] * step).sum() - slope) <= 1e-6 * (np.abs(exact[i][0] * step).sum() + 1.0), name      # the formula's own gradient
        # the call's: its tolerance, and what the roundings of the saved out and lse change
        allowed = ((want[i][1] + np.abs(want[i][0] - exact[i][0])) * np.abs(step)).sum()
        assert abs((host_f64(got) * step).sum() - slope) <= allowed + 1e-6 * np.abs(exact[i][0] * step).sum(), name


def test_streams_and_graph(sp):
    """A forward and a backward on another stream, and both captured into a graph that is replayed with other inputs."""
    import torch
    B, s, off, Hq, Hkv, D, L, top_k = 1, 300, 468, 4, 2, 64, 64, 4
    N = off + s
    sets = [tensors(B, s, N, Hq, Hkv, D, salt=40 + i)[0] for i in range(3)]
    idxs = [torch.from_numpy(random_index(np.random.default_rng(i), B, Hq, s, top_k, -(-N // L), False)).cuda() for i in range(3)]

    def step(t, idx, ws):
        means = sp.slimpipe_attn_block_means(t["k"], 0, N, L)
        chosen = sp.slimpipe_attn_block_select(t["q"], means, off, 0, N, L, top_k)
        o, l = sp.slimpipe_attn_block_fwd(t["q"], t["k"], t["v"], chosen, off, 0, N, L, workspace=ws[0])
        o, l = sp.slimpipe_attn_block_fwd(t["q"], t["k"], t["v"], idx, off, 0, N, L, workspace=ws[0])
        dk, dv = torch.zeros((2,) + t["k"].shape, device="cuda")
        dq = sp.slimpipe_attn_block_bwd(t["q"], t["k"], t["v"], idx, o, t["do"], l, off, 0, N, L, dk, dv, workspace=ws[1])
        return chosen, o, l, dq, dk, dv
    ws = [torch.empty(sp.slimpipe_attn_block_workspace_bytes(sets[0]["q"], sets[0]["k"], idxs[0], off, 0, N, L, True, bwd), device="cuda", dtype=torch.uint8)
          for bwd in (False, True)]
    eager = [step(t, i, ws) for t, i in zip(sets, idxs)]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        again = step(sets[1], idxs[1], ws)
    other.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(again, eager[1]))
    buf, ibuf = {k: v.clone() for k, v in sets[0].items()}, idxs[0].clone()
    graph = torch.cuda.CUDAGraph()
    sp.slimpipe_attn_init()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(buf, ibuf, ws)
    for i in (1, 2, 0, 2):
        for k in buf:
            buf[k].copy_(sets[i][k])
        ibuf.copy_(idxs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, eager[i])), i
        step(sets[0], idxs[0], ws)
        torch.cuda.synchronize()
