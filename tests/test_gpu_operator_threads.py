"""Two host threads at once, a stream each: every call comes to its end, with the results that it has alone."""
import threading

import pytest

from gpu_util import dev_bf16
from synth_inputs import normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def in_threads(work, n, times):
    """work(i) `times` times in each of n threads -> the results that differ from a first run, exceptions, and the rounds that each thread has done."""
    import torch
    want = [work(i) for i in range(n)]
    torch.cuda.synchronize()
    wrong, raised, done = [], [], [0] * n

    def run(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(times):
                    got = work(i)
                    stream.synchronize()
                    if not all(torch.equal(x, y) for x, y in zip(got, want[i])):
                        wrong.append(i)
                    done[i] += 1
        except BaseException as e:                            # (one that ends a thread is lost otherwise)
            raised.append((i, e))
    threads = [threading.Thread(target=run, args=(i,)) for i in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return wrong, raised, done


def test_every_round_of_two_threads(sp):
    import torch
    s, off, Hq, Hkv, D, L, top_k = 300, 700, 8, 2, 128, 64, 5
    N = off + s
    sets = []
    for i in range(2):
        q, k, v, do = (dev_bf16(normal_bf16((1, n, h, D), 43, tag, i)) for tag, n, h in (("q", s, Hq), ("k", N, Hkv), ("v", N, Hkv), ("do", s, Hq)))
        cache = sp.KvCache4.empty(1, N, Hkv, D)
        sets.append((q, k, v, do, cache))

    def work(i):
        q, k, v, do, cache = sets[i]
        index = sp.slimpipe_attn_block_select(q, sp.slimpipe_attn_block_means(k, 0, N, L), off, 0, N, L, top_k)
        out, lse = sp.slimpipe_attn_block_fwd(q, k, v, index, off, 0, N, L)
        few = sp.slimpipe_attn_block_fwd(q[:, :2], k, v, index[:, :, :2].contiguous(), off, 0, N, L)
        dk, dv = torch.zeros((2,) + k.shape, device="cuda")
        dq = sp.slimpipe_attn_block_bwd(q, k, v, index, out, do, lse, off, 0, N, L, dk, dv)
        sp.slimpipe_attn_kv4_store(k, v, cache, 0)
        return index, out, lse, *few, dq, dk, dv, *sp.slimpipe_attn_kv4_load(cache, 0, N), *sp.slimpipe_attn_fwd_kv4(q, cache, off, 0, N), \
            *sp.slimpipe_attn_fwd_kv4(q[:, :1], cache, off, 0, N)
    wrong, raised, done = in_threads(work, 2, 20)
    assert not raised and not wrong and done == [20, 20], (wrong, raised, done)
