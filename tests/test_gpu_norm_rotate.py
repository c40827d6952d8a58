"""Norm and rotation of queries and keys on the GPU against plain 64-bit definitions: results, gradients, strides, what stays untouched.

Tolerances.  A result is rounded to bf16 once: at most 2^-8 of its size.  Before that come norms and products in 32 bits (a few dozen roundings of 2^-24)
and a sine and cosine, which have to keep within 2^-16 of the definition for the pair not to show it: 2^-15 of the pair's sizes in all."""
import numpy as np
import pytest

from gpu_util import host_f64, say

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def frequencies(rotate, base=10000.0):
    return base ** (-2.0 * np.arange(rotate // 2) / max(rotate, 1))


def pairs(rotate, interleaved):
    i = np.arange(rotate // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotate // 2)


def turned(x, pos, freq, interleaved, sign=1.0):
    a, b = pairs(2 * len(freq), interleaved)
    # (the angle as a fraction of a turn in extended precision: positions up to 2^40 here)
    angle = (np.longdouble(pos)[..., None] * np.longdouble(freq)).astype(np.longdouble)
    c, s = np.cos(angle).astype(np.float64)[:, :, None], sign * np.sin(angle).astype(np.float64)[:, :, None]
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def forward(x, w, pos, freq, interleaved):
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w
    return y, turned(y, pos, freq, interleaved)


def backward(x, w, dz, pos, freq, interleaved):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    dy = turned(dz, pos, freq, interleaved, -1.0)
    n, g = x * r, dy * w
    return r * (g - n * (g * n).mean(-1, keepdims=True)), (dy * n).sum((0, 1, 2))


def room(y, rotate, interleaved):
    """What an element may be off beside the rounding of the result."""
    size = np.abs(y)
    a, b = pairs(rotate, interleaved)
    size[..., a] = size[..., b] = size[..., a] + size[..., b]
    return 2.0 ** -15 * size + 1e-30


def fits(ok):
    """(A comparison of whole arrays in an assert would print them.)"""
    return bool(ok.all())


def tensors(B, s, Hq, Hkv, D, seed, fused=True):
    """q and k as parts of a projected row with values behind them, and two weights."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, s, Hq + 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    w = 1.0 + 0.25 * torch.randn((2, D), generator=g, device="cuda")
    return x, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], w[0].clone(), w[1].clone()


SHAPES = [
    # B, s, Hq, Hkv, D, rotate, interleaved, first position
    (1, 1, 1, 1, 64, 64, False, 0),
    (1, 1, 40, 40, 128, 128, False, 130700),
    (4, 1, 8, 1, 128, 128, False, 5),
    (2, 7, 8, 1, 128, 128, True, 1000003),
    (1, 9, 12, 4, 64, 32, False, 77),
    (3, 33, 12, 4, 64, 16, True, 4096),
    (1, 17, 5, 3, 64, 64, True, 3),
    (2, 65, 3, 1, 128, 64, False, 2 ** 31 + 5),
    (1, 129, 16, 16, 128, 32, False, 2 ** 40 + 1),
    (1, 300, 8, 2, 128, 0, False, 9),
    (1, 2049, 4, 4, 64, 64, False, 100),
    (5, 401, 8, 1, 128, 112, False, 100),
]


def positions_of(B, s, first):
    return np.broadcast_to(first + np.arange(s), (B, s))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("apart,weighted", [(False, True), (True, False)])
def test_forward(sp, shape, apart, weighted):
    import torch
    B, s, Hq, Hkv, D, rotate, interleaved, first = shape
    say("norm_rotate forward %r apart=%d weighted=%d" % (shape, apart, weighted))
    x, q, k, wq, wk = tensors(B, s, Hq, Hkv, D, 3)
    freq = frequencies(rotate)
    pos, at = positions_of(B, s, first), first
    if apart:
        pos = pos + 13 * np.arange(B)[:, None]
        at = torch.from_numpy(pos.copy()).cuda()
    got = sp.slimpipe_attn_norm_rotate(q, k, wq if weighted else None, wk if weighted else None, torch.from_numpy(freq).cuda(), at, EPS, interleaved)
    for z, src, w in zip(got, (q, k), (wq, wk)):
        y, want = forward(host_f64(src), host_f64(w) if weighted else np.ones(D), pos, freq, interleaved)
        z = host_f64(z)
        assert np.isfinite(z).all()
        assert fits(np.abs(z - want) <= 2.0 ** -8 * np.abs(want) + room(y, rotate, interleaved))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("f32", [(False, True), (True, False)])
def test_backward(sp, shape, f32):
    import torch
    B, s, Hq, Hkv, D, rotate, interleaved, first = shape
    say("norm_rotate backward %r f32=%r" % (shape, f32))
    x, q, k, wq, wk = tensors(B, s, Hq, Hkv, D, 4)
    freq = frequencies(rotate)
    pos = positions_of(B, s, first)
    g = torch.Generator(device="cuda").manual_seed(5)
    dz = [torch.randn(t.shape, generator=g, device="cuda").to(torch.float32 if f else torch.bfloat16) for t, f in zip((q, k), f32)]
    args = (q, k, wq, wk, torch.from_numpy(freq).cuda(), first, dz[0], dz[1], EPS, interleaved)
    got = sp.slimpipe_attn_norm_rotate_bwd(*args)
    again = sp.slimpipe_attn_norm_rotate_bwd(*args)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for i, (src, w) in enumerate(((q, wq), (k, wk))):
        xs = host_f64(src)
        dx, dw = backward(xs, host_f64(w), host_f64(dz[i]), pos, freq, interleaved)
        # dx = r (g - n mean(g n)): off by a bf16 rounding, and by 2^-15 of what is added up in it
        r = 1.0 / np.sqrt((xs * xs).mean(-1, keepdims=True) + EPS)
        size = np.abs(turned(host_f64(dz[i]), pos, freq, interleaved, -1.0)) * np.abs(host_f64(w))
        a, b = pairs(rotate, interleaved)
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
        size = 2 * r * (size + np.abs(xs * r) * size.mean(-1, keepdims=True))
        z = host_f64(got[i])
        assert fits(np.abs(z - dx) <= 2.0 ** -8 * np.abs(dx) + 2.0 ** -15 * size)
        # a sum of n terms of about 1, in 32 bits with 2^-15 a term at worst, all of one sign only if the sines' errors are
        n = xs.shape[0] * xs.shape[1] * xs.shape[2]
        assert fits(np.abs(host_f64(got[2 + i]) - dw) <= 2.0 ** -15 * 2 * n ** 0.5 + 2.0 ** -17 * n)


def test_gradient_against_differences(sp):
    """Gradients against central differences of the 64-bit definition."""
    import torch
    B, s, Hq, Hkv, D, rotate = 1, 3, 2, 1, 64, 32
    say("norm_rotate differences")
    x, q, k, wq, wk = tensors(B, s, Hq, Hkv, D, 8)
    freq, pos = frequencies(rotate), positions_of(B, s, 11)
    g = torch.Generator(device="cuda").manual_seed(9)
    dz = [torch.randn(t.shape, generator=g, device="cuda") for t in (q, k)]
    dq, dk, dwq, dwk = sp.slimpipe_attn_norm_rotate_bwd(q, k, wq, wk, torch.from_numpy(freq).cuda(), 11, dz[0], dz[1], EPS)
    rng = np.random.RandomState(1)
    for src, w, d, dx, dw in ((q, wq, dz[0], dq, dwq), (k, wk, dz[1], dk, dwk)):
        x0, w0, d0 = host_f64(src), host_f64(w), host_f64(d)
        for _ in range(4):
            ux, uw = rng.randn(*x0.shape), rng.randn(*w0.shape)
            h = 1e-5
            f = [(forward(x0 + t * ux, w0 + t * uw, pos, freq, False)[1] * d0).sum() for t in (h, -h)]
            want = (f[0] - f[1]) / (2 * h)
            dx64, dw64 = host_f64(dx), host_f64(dw)
            got = (dx64 * ux).sum() + (dw64 * uw).sum()
            # roundings of dx to bf16, each with the direction's element: all of one sign at worst
            assert abs(got - want) <= 2.0 ** -8 * np.abs(dx64 * ux).sum() + 2.0 ** -12 * np.abs(dw64 * uw).sum() + 1e-6 * abs(want)


def test_weight_gradients_added_over_slices(sp):
    import torch
    say("norm_rotate weights over slices")
    x, q, k, wq, wk = tensors(2, 96, 8, 2, 128, 12)
    f = torch.from_numpy(frequencies(128)).cuda()
    dz = [torch.randn(t.shape, device="cuda") for t in (q, k)]
    whole = sp.slimpipe_attn_norm_rotate_bwd(q, k, wq, wk, f, 0, dz[0], dz[1], EPS)
    sums = [torch.full((128,), 7.0, device="cuda") for _ in range(2)]
    for i, r in enumerate((slice(0, 32), slice(32, 96))):
        part = sp.slimpipe_attn_norm_rotate_bwd(q[:, r], k[:, r], wq, wk, f, r.start, dz[0][:, r], dz[1][:, r], EPS, dq_weight=sums[0], dk_weight=sums[1],
                                                weight_accumulate=i > 0)
        assert torch.equal(part[0], whole[0][:, r]) and torch.equal(part[1], whole[1][:, r])
    for a, b, n in zip(sums, whole[2:], (2 * 96 * 8, 2 * 96 * 2)):
        assert (a - b).abs().max() <= 2.0 ** -22 * 4 * n      # (sums of n terms of up to 4 in two orders)


def test_in_place_and_into_a_prefix(sp):
    """Results over their operands, and keys straight into rows of a prefix, whose other rows stay."""
    import torch
    say("norm_rotate in place")
    x, q, k, wq, wk = tensors(2, 50, 8, 2, 128, 21)
    f = torch.from_numpy(frequencies(128)).cuda()
    want = sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 100, EPS)
    prefix = torch.full((2, 170, 2, 128), -3.0, device="cuda", dtype=torch.bfloat16)
    got = sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 100, EPS, k_out=prefix[:, 100:150])
    assert torch.equal(got[0], want[0]) and torch.equal(prefix[:, 100:150], want[1])
    assert (prefix[:, :100] == -3.0).all() and (prefix[:, 150:] == -3.0).all()
    values = x[:, :, 10:].clone()
    sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 100, EPS, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, 10:], values)


def test_one_side_alone(sp):
    import torch
    say("norm_rotate one side")
    x, q, k, wq, wk = tensors(1, 21, 4, 2, 64, 22)
    f = torch.from_numpy(frequencies(64)).cuda()
    both = sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 7, EPS)
    none = q[:, :, :0]
    assert torch.equal(sp.slimpipe_attn_norm_rotate(q, none, wq, None, f, 7, EPS)[0], both[0])
    assert torch.equal(sp.slimpipe_attn_norm_rotate(none, k, None, wk, f, 7, EPS)[1], both[1])
    g = torch.randn(q.shape, device="cuda"), torch.randn(k.shape, device="cuda")
    grads = sp.slimpipe_attn_norm_rotate_bwd(q, k, wq, wk, f, 7, g[0], g[1], EPS)
    alone = sp.slimpipe_attn_norm_rotate_bwd(none, k, None, wk, f, 7, g[0][:, :, :0], g[1], EPS)
    assert torch.equal(alone[1], grads[1])
    # (other workgroups, another order of 42 terms of up to 16)
    assert (alone[3] - grads[3]).abs().max() <= 42 * 16 * 2.0 ** -22


def test_zero_rows_and_values_that_are_not_finite(sp):
    """A row of zeros stays one and has finite gradients; a NaN or an infinity stays with its head."""
    import torch
    say("norm_rotate special values")
    x, q, k, wq, wk = tensors(1, 16, 4, 2, 128, 23)
    f = torch.from_numpy(frequencies(64)).cuda()
    clean = [t.clone() for t in sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 7, EPS)]
    q[0, 3, 1] = 0.0
    q[0, 4, 2, 5] = float("nan")
    k[0, 15, 1, 127] = float("inf")
    got = sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 7, EPS)
    assert (got[0][0, 3, 1] == 0).all() and torch.isnan(got[0][0, 4, 2]).all() and torch.isnan(got[1][0, 15, 1, 127])
    for z, c, touched in ((got[0], clean[0], [(3, 1), (4, 2)]), (got[1], clean[1], [(15, 1)])):
        same = (z == c).all(-1)[0]
        for t in touched:
            same[t] = True
        assert same.all()
    d = torch.randn(q.shape, device="cuda"), torch.randn(k.shape, device="cuda")
    dq, dk, _, _ = sp.slimpipe_attn_norm_rotate_bwd(q, k, None, None, f, 7, d[0], d[1], EPS)
    bad = ~torch.isfinite(dq.float()).all(-1)[0]
    assert bad[4, 2] and bad.sum() == 1 and (~torch.isfinite(dk.float()).all(-1)[0]).sum() == 1
    # of the row of zeros: g / sqrt(eps)
    assert torch.isfinite(dq[0, 3, 1].float()).all() and dq[0, 3, 1].abs().max() > 100


def test_smallest_eps_and_rows_of_zeros(sp):
    import torch
    x, q, k, wq, wk = tensors(1, 8, 4, 2, 64, 25)
    q[0, 2] = 0.0
    f = torch.from_numpy(frequencies(64)).cuda()
    eps = 2.0 ** -126
    out = sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, 7, eps)
    assert (out[0][0, 2] == 0).all() and all(torch.isfinite(t.float()).all() for t in out)
    dq = sp.slimpipe_attn_norm_rotate_bwd(q, k, wq, wk, f, 7, torch.zeros_like(q), torch.zeros_like(k), eps)[0]
    assert (dq == 0).all()


def test_captured(sp):
    """Both directions in a captured graph, replayed on other inputs, against eager calls."""
    import torch
    say("norm_rotate graph")
    sp.slimpipe_attn_init()
    x, q, k, wq, wk = tensors(2, 40, 8, 2, 128, 31)
    f = torch.from_numpy(frequencies(128)).cuda()
    at = torch.arange(80, device="cuda").reshape(2, 40)
    d = torch.randn(q.shape, device="cuda"), torch.randn(k.shape, device="cuda")
    ws = torch.empty(sp.slimpipe_attn_norm_rotate_workspace_bytes(q, k), device="cuda", dtype=torch.uint8)
    out = [torch.empty(t.shape, device="cuda", dtype=torch.bfloat16) for t in (q, k)]
    grads = [torch.empty_strided(t.shape, t.stride(), device="cuda", dtype=torch.bfloat16) for t in (q, k)] + [torch.empty(128, device="cuda") for _ in "qk"]

    def calls():
        sp.slimpipe_attn_norm_rotate(q, k, wq, wk, f, at, EPS, q_out=out[0], k_out=out[1])
        sp.slimpipe_attn_norm_rotate_bwd(q, k, wq, wk, f, at, d[0], d[1], EPS, dq=grads[0], dk=grads[1], dq_weight=grads[2], dk_weight=grads[3], workspace=ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for n in range(3):
        x.normal_()
        at.add_(1000 * n)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out + grads]
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, out + grads))


def test_training_over_slices(sp):
    """Norm, rotation and attention of a sequence cut into slices, forward and backward through the calls as a training step makes them, against 64-bit
    automatic differentiation of the whole sequence.  Queries, keys, outputs, dq and dS are bf16 on the way: gradients within 2e-2 of their norm, the bar of the attention's
    own gradients."""
    import torch
    say("norm_rotate, attention, two slices")
    B, n, slices, Hq, Hkv, D = 2, 128, 2, 4, 2, 64
    step = n // slices
    x, q, k, wq, wk = tensors(B, n, Hq, Hkv, D, 41)
    v = x[:, :, Hq + Hkv:].contiguous()
    freq = torch.from_numpy(frequencies(D)).cuda()
    do = torch.randn(q.shape, device="cuda").to(torch.bfloat16)
    prefix = torch.zeros(k.shape, device="cuda", dtype=torch.bfloat16)
    saved = []
    for i in range(slices):
        r = slice(i * step, (i + 1) * step)
        turned, _ = sp.slimpipe_attn_norm_rotate(q[:, r], k[:, r], wq, wk, freq, r.start, EPS, k_out=prefix[:, r])
        saved.append((r, turned) + sp.slimpipe_attn_fwd(turned, prefix, v, r.start, 0, r.stop))
    dk, dv = torch.zeros((2,) + k.shape, device="cuda")
    dx = torch.zeros_like(x)
    dw = [torch.zeros(D, device="cuda") for _ in range(2)]
    for r, turned, out, lse in reversed(saved):
        dq = sp.slimpipe_attn_bwd(turned, prefix, v, out, do[:, r], lse, r.start, 0, r.stop, dk, dv)
        sp.slimpipe_attn_norm_rotate_bwd(q[:, r], k[:, r], wq, wk, freq, r.start, dq, dk[:, r], EPS, dq=dx[:, r, :Hq], dk=dx[:, r, Hq:Hq + Hkv],
                                         dq_weight=dw[0], dk_weight=dw[1], weight_accumulate=True)
    leaf = [t.detach().cpu().double().requires_grad_() for t in (q, k, v, wq, wk)]
    angle = torch.arange(n, dtype=torch.float64)[:, None] * freq.cpu()
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turn(t, w):
        y = t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS) * w
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat((a * c - b * s, b * c + a * s), -1)
    qq, kk = turn(leaf[0], leaf[3]), turn(leaf[1], leaf[4]).repeat_interleave(Hq // Hkv, 2)
    vv = leaf[2].repeat_interleave(Hq // Hkv, 2)
    score = (qq.transpose(1, 2) @ kk.permute(0, 2, 3, 1).contiguous()) / D ** 0.5
    score = score.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf"))
    out = (score.softmax(-1) @ vv.transpose(1, 2)).transpose(1, 2)
    (out * do.cpu().double()).sum().backward()
    got = [dx[:, :, :Hq], dx[:, :, Hq:Hq + Hkv], dv, dw[0], dw[1]]
    for g, t in zip(got, leaf):
        g = torch.from_numpy(host_f64(g))
        assert float((g - t.grad).norm() / t.grad.norm()) <= 2e-2
