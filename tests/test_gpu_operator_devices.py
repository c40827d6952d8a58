"""Sparse attention and the 4-bit cache, given one tensor that is not on the GPU: refused before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu

S, HQ, H, D, N, L, K = 4, 8, 2, 64, 256, 64, 2


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def tensors():
    import torch
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device="cuda")
    return dict(q=t(1, S, HQ, D), k=t(1, N, H, D), v=t(1, N, H, D), out=t(1, S, HQ, D), d_out=t(1, S, HQ, D), lse=t(1, HQ, S, dtype=f32),
                index=t(1, HQ, S, K, dtype=i32), dq=t(1, S, HQ, D), dk=t(1, N, H, D, dtype=f32), dv=t(1, N, H, D, dtype=f32), means=t(1, H, N // L, D, dtype=f32),
                k_codes=t(1, N, H, D // 2, dtype=u8), k_scales=t(1, N, H, D // 32, dtype=u8), v_codes=t(1, N, H, D // 2, dtype=u8),
                v_scales=t(1, N, H, D // 32, dtype=u8), k_rows=t(1, S, H, D), v_rows=t(1, S, H, D), ws=t(1 << 22, dtype=u8))


def cache(sp, a):
    return sp.KvCache4(a["k_codes"], a["k_scales"], a["v_codes"], a["v_scales"])


CACHE = "k_codes k_scales v_codes v_scales"
CALLS = [
    ("k means", lambda sp, a: sp.slimpipe_attn_block_means(a["k"], 0, N, L, means=a["means"])),
    ("q means index", lambda sp, a: sp.slimpipe_attn_block_select(a["q"], a["means"], 0, 0, N, L, K, index=a["index"])),
    ("q k v index out lse ws", lambda sp, a: sp.slimpipe_attn_block_fwd(a["q"], a["k"], a["v"], a["index"], 0, 0, N, L, out=a["out"], lse=a["lse"], workspace=a["ws"])),
    ("q k v index out d_out lse dk dv dq ws", lambda sp, a: sp.slimpipe_attn_block_bwd(a["q"], a["k"], a["v"], a["index"], a["out"], a["d_out"], a["lse"], 0, 0, N, L,
                                                                                        a["dk"], a["dv"], dq=a["dq"], workspace=a["ws"])),
    ("k_rows v_rows " + CACHE, lambda sp, a: sp.slimpipe_attn_kv4_store(a["k_rows"], a["v_rows"], cache(sp, a), 0)),
    ("k_rows v_rows " + CACHE, lambda sp, a: sp.slimpipe_attn_kv4_load(cache(sp, a), 0, S, k_rows=a["k_rows"], v_rows=a["v_rows"])),
    ("q out lse ws " + CACHE, lambda sp, a: sp.slimpipe_attn_fwd_kv4(a["q"], cache(sp, a), 0, 0, N, out=a["out"], lse=a["lse"], workspace=a["ws"])),
]


@pytest.mark.parametrize("at", range(len(CALLS)))
def test_one_tensor_on_the_host(sp, at):
    import torch
    names, call = CALLS[at]
    a = tensors()
    call(sp, a)                                              # all of them on the GPU
    torch.cuda.synchronize()
    for name in names.split():
        with pytest.raises(sp.SlimpipeError):
            call(sp, {**a, name: a[name].cpu()})


def test_a_chunk_on_the_host(sp):
    a = tensors()
    lists = {n: [a[n], a[n].clone()] for n in ("k", "v", "dk", "dv")}
    means = a["means"].repeat(1, 1, 2, 1)
    for name in lists:
        x = {**lists, name: [lists[name][0], lists[name][1].cpu()]}
        if name == "k":
            with pytest.raises(sp.SlimpipeError):
                sp.slimpipe_attn_block_means(x["k"], 0, N, L, means=means)
        if name in "kv":
            with pytest.raises(sp.SlimpipeError):
                sp.slimpipe_attn_block_fwd(a["q"], x["k"], x["v"], a["index"], 0, 0, N, L)
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_bwd(a["q"], x["k"], x["v"], a["index"], a["out"], a["d_out"], a["lse"], 0, 0, N, L, x["dk"], x["dv"])
