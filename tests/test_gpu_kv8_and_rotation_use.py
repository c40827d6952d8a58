"""The 8-bit cache, eviction from it and the norm and rotation in use: tensors that are not on the GPU, two host threads, memory around results, offsets that
pass 32 bits, two captured steps that share a workspace."""
import math

import pytest

from gpu_util import dev_bf16, say
from synth_inputs import normal_bf16
from test_gpu_operator_threads import in_threads
import test_host_kv8_and_rotation as host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


@pytest.mark.parametrize("i", range(len(host.WRAPPED)))
def test_one_tensor_on_the_host(sp, i):
    import torch
    names, call = host.WRAPPED[i]
    a = {k: v.cuda() for k, v in host.right().items()}
    call(sp, a)                                              # all of them on the GPU
    torch.cuda.synchronize()
    for name in names.split():
        with pytest.raises(sp.SlimpipeError):
            call(sp, {**a, name: a[name].cpu()})


def test_every_round_of_two_threads(sp):
    import torch
    s, off, Hq, Hkv, D, L = 300, 700, 8, 2, 128, 64
    N, keep = off + s, 400
    freq = torch.pow(10000.0, -2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    w = torch.ones(D, device="cuda")
    sets = []
    for i in range(2):
        q, k, v = (dev_bf16(normal_bf16((1, n, h, D), 63, tag, i)) for tag, n, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv)))
        sets.append((q, k, v, sp.KvCache8.empty(1, N, Hkv, D, L), sp.KvCache8.empty(1, keep, Hkv, D, L)))

    def work(i):
        q, k, v, cache, kept = sets[i]
        turned = sp.slimpipe_attn_norm_rotate(q, k[:, off:], w, w, freq, off)
        grads = sp.slimpipe_attn_norm_rotate_bwd(q, k[:, off:], w, w, freq, off, *turned)
        sp.slimpipe_attn_kv8_store(k, v, cache, 0)
        out, lse = sp.slimpipe_attn_fwd_kv8(q, cache, off, 0, N)
        few = sp.slimpipe_attn_fwd_kv8(q[:, :1], cache, off, 0, N)
        sums = sp.slimpipe_attn_kv8_weights(q, cache, lse, off, 0, N)
        index = sp.slimpipe_attn_kv8_keep(sums, N, keep, 10)
        sp.slimpipe_attn_kv8_gather(cache, index, kept)
        return (*turned, *grads, out, lse, *few, sums, index, *sp.slimpipe_attn_kv8_load(kept, 0, keep))
    wrong, raised, done = in_threads(work, 2, 20)
    assert not raised and not wrong and done == [20, 20], (wrong, raised, done)


def guarded(shape, dtype, fill):
    """A contiguous tensor inside a larger allocation full of `fill` -> (tensor, check that nothing around it has changed)."""
    import torch
    n = math.prod(shape)
    pad = 4096 // torch.empty((), dtype=dtype).element_size()
    whole = torch.full((n + 2 * pad,), fill, device="cuda", dtype=dtype)
    return whole[pad:pad + n].view(shape), lambda: bool((whole[:pad] == fill).all() and (whole[pad + n:] == fill).all())


@pytest.mark.parametrize("B,s,off,Hq,Hkv,D,L", [(1, 1, 5000, 8, 1, 128, 64), (2, 3, 777, 12, 4, 64, 16), (1, 130, 333, 6, 2, 64, 128), (1, 600, 700, 4, 2, 128, 256), (1, 1100, 700, 4, 2, 64, 64), (4, 200, 1500, 16, 16, 64, 16)])
def test_memory_around_results(sp, B, s, off, Hq, Hkv, D, L):
    import torch
    say("guards %r" % ((B, s, off, Hq, Hkv, D, L),))
    N, keep = off + s, (off + s) // 3
    q, k, v = (dev_bf16(normal_bf16((B, n, h, D), 64, tag)) for tag, n, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv)))
    freq = torch.pow(10000.0, -2.0 * torch.arange(D // 4, device="cuda", dtype=torch.float64) / D * 2)
    w = torch.ones(D, device="cuda")
    checks = []

    def room(shape, dtype, fill=77):
        x, ok = guarded(shape, dtype, fill)
        checks.append(ok)
        return x

    def cache(n):
        blocks = -(-n // L)
        return sp.KvCache8(room((B, n, Hkv, D), torch.uint8), room((B, blocks, Hkv), torch.uint8), room((B, n, Hkv, D), torch.uint8),
                           room((B, blocks, Hkv), torch.uint8), L)
    q_out, k_out = room(q.shape, torch.bfloat16), room(k.shape, torch.bfloat16)
    sp.slimpipe_attn_norm_rotate(q, k[:, :s], w, w, freq, 5, q_out=q_out, k_out=k_out[:, :s])
    assert (k_out[:, s:] == 77).all()
    ws = room((sp.slimpipe_attn_norm_rotate_workspace_bytes(q, k[:, :s]),), torch.uint8)
    sp.slimpipe_attn_norm_rotate_bwd(q, k[:, :s], w, w, freq, 5, q_out, k_out[:, :s], dq=room(q.shape, torch.bfloat16), dk=room(k.shape, torch.bfloat16)[:, :s],
                                     dq_weight=room((D,), torch.float32), dk_weight=room((D,), torch.float32), workspace=ws)
    one, two = cache(N), cache(keep)
    sp.slimpipe_attn_kv8_store(k[:, :off], v[:, :off], one, 0)
    sp.slimpipe_attn_kv8_store(k[:, off:], v[:, off:], one, off)
    sp.slimpipe_attn_kv8_load(one, 0, N, k_rows=room(k.shape, torch.bfloat16), v_rows=room(k.shape, torch.bfloat16))
    lse = room((B, Hq, s), torch.float32)
    ws = room((sp.slimpipe_attn_kv8_workspace_bytes(q, one, off, 0, N),), torch.uint8)
    sp.slimpipe_attn_fwd_kv8(q, one, off, 0, N, out=room(q.shape, torch.bfloat16), lse=lse, workspace=ws)
    sums = room((B, Hkv, N), torch.float32)
    ws = room((sp.slimpipe_attn_kv8_weights_workspace_bytes(q, one, off, 0, N),), torch.uint8)
    sp.slimpipe_attn_kv8_weights(q, one, lse, off, 0, N, weights=sums, workspace=ws)
    index = room((B, Hkv, keep), torch.int32)
    sp.slimpipe_attn_kv8_keep(sums, N, keep, min(9, keep), index=index)
    sp.slimpipe_attn_kv8_gather(one, index, two, sums, room((B, Hkv, keep), torch.float32))
    torch.cuda.synchronize()
    assert all(ok() for ok in checks)


def test_offsets_that_pass_32_bits(sp):
    """Rows behind 2^32 bytes of codes give what the same rows at the start of a small cache give."""
    import torch
    H, Hq, D, L, base, n = 8, 16, 128, 64, 1 << 22, 600
    N = base + n
    big = sp.KvCache8(*(torch.empty(shape, device="cuda", dtype=torch.uint8) for shape in ((1, N, H, D), (1, -(-N // L), H)) * 2), L)
    small = sp.KvCache8.empty(1, n, H, D, L)
    k, v = (dev_bf16(normal_bf16((1, n, H, D), 65, tag)) for tag in "kv")
    for part in (slice(0, 330), slice(330, n)):
        sp.slimpipe_attn_kv8_store(k[:, part], v[:, part], big, base + part.start)
        sp.slimpipe_attn_kv8_store(k[:, part], v[:, part], small, part.start)
    for x, y in zip(sp.slimpipe_attn_kv8_load(big, base, N), sp.slimpipe_attn_kv8_load(small, 0, n)):
        assert torch.equal(x, y)
    sums = torch.zeros((1, H, N), device="cuda")
    for s in (1, 200, 550):
        q = dev_bf16(normal_bf16((1, s, Hq, D), 65, "q", s))
        a = sp.slimpipe_attn_fwd_kv8(q, big, N - s, base, N)
        b = sp.slimpipe_attn_fwd_kv8(q, small, n - s, 0, n)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        sp.slimpipe_attn_kv8_weights(q, big, a[1], N - s, base, N, weights=sums, previous=sums)
        got = sp.slimpipe_attn_kv8_weights(q, big, a[1], N - s, base, N)[..., base:]
        assert torch.equal(got, sp.slimpipe_attn_kv8_weights(q, small, b[1], n - s, 0, n))
    index = sp.slimpipe_attn_kv8_keep(sums, N, 300, 20)
    assert (index >= base).all() and (index[..., 1:] > index[..., :-1]).all() and (index[..., -20:] == torch.arange(N - 20, N, device="cuda")).all()
    kept = sp.slimpipe_attn_kv8_gather(big, index, sp.KvCache8.empty(1, 300, H, D, L))
    want = sp.slimpipe_attn_kv8_gather(small, (index - base).int().contiguous(), sp.KvCache8.empty(1, 300, H, D, L))
    assert all(torch.equal(x, y) for x, y in zip(kept[:4], want[:4]))


def test_two_graphs_that_share_a_workspace(sp):
    """Replayed one after the other on a stream, in turn, with eager calls between."""
    import torch
    sp.slimpipe_attn_init()
    B, Hq, Hkv, D, L, N = 1, 8, 2, 128, 64, 3000
    k, v = (dev_bf16(normal_bf16((B, N, Hkv, D), 66, tag)) for tag in "kv")
    cache = sp.KvCache8.empty(B, N, Hkv, D, L)
    sp.slimpipe_attn_kv8_store(k, v, cache, 0)
    qs = [dev_bf16(normal_bf16((B, s, Hq, D), 66, "q", s)) for s in (1, 600)]
    need = max(max(sp.slimpipe_attn_kv8_workspace_bytes(q, cache, N - q.shape[1], 0, N), sp.slimpipe_attn_kv8_weights_workspace_bytes(q, cache, N - q.shape[1], 0, N))
               for q in qs)
    ws = torch.empty(need, device="cuda", dtype=torch.uint8)
    out = [torch.empty_like(q) for q in qs]
    lse = [torch.empty((B, Hq, q.shape[1]), device="cuda") for q in qs]
    sums = [torch.zeros((B, Hkv, N), device="cuda") for _ in qs]

    def step(i):
        off = N - qs[i].shape[1]
        sp.slimpipe_attn_fwd_kv8(qs[i], cache, off, 0, N, out=out[i], lse=lse[i], workspace=ws)
        sp.slimpipe_attn_kv8_weights(qs[i], cache, lse[i], off, 0, N, weights=sums[i], workspace=ws)
    want = []
    for i in range(2):
        step(i)
        want.append([x.clone() for x in (out[i], lse[i], sums[i])])
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i)
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        for x in (out[i], lse[i], sums[i]):
            x.zero_()
        graphs[i].replay()
        step(1 - i)
        torch.cuda.synchronize()
        for j in range(2):
            assert all(torch.equal(x, y) for x, y in zip((out[j], lse[j], sums[j]), want[j]))
