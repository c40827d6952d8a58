"""CPU-only checks of sparse attention over key blocks and of the 4-bit cache at the boundary: what is refused, with which code, before
anything touches a device; workspace sizes."""
import ctypes

import pytest

NULL, SHAPE, RANGE, STRIDE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5, -6


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def params(sp, **change):
    p = sp.AttnParams()
    p.batch, p.s_q, p.n_q_heads, p.n_kv_heads, p.head_dim, p.causal = 1, 512, 8, 1, 128, 1
    p.kv_capacity, p.q_offset, p.kv_begin, p.kv_end = 4096, 1024, 0, 1536
    p.scale, p.out_dtype = 0.088, sp.BF16
    p.q_stride_b, p.q_stride_s, p.q_stride_h = 512 * 8 * 128, 8 * 128, 128
    p.kv_stride_b, p.kv_stride_s, p.kv_stride_h = 4096 * 128, 128, 128
    p.o_stride_b, p.o_stride_s, p.o_stride_h = 512 * 8 * 128, 8 * 128, 128
    p.do_stride_b, p.do_stride_s, p.do_stride_h = 512 * 8 * 128, 8 * 128, 128
    for k, v in change.items():
        setattr(p, k, v)
    return p


A, ODD = 0x1000, 0x1008            # addresses that are never read: a call is refused first
WS = 1 << 50


def table(*ptrs):
    return (ctypes.c_void_p * len(ptrs))(*ptrs)


def means(sp, p, k=(A,), chunk_len=4096, block=64, out=A):
    return sp.lib.slimpipe_attn_block_means(ctypes.byref(p), table(*k), len(k), chunk_len, block, out, None)


def select(sp, p, q=A, m=A, block=64, top_k=4, index=A):
    return sp.lib.slimpipe_attn_block_select(ctypes.byref(p), q, m, block, top_k, index, None)


def fwd(sp, p, q=A, k=(A,), v=(A,), chunk_len=4096, block=64, top_k=4, index=A, out=A, lse=A, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_block_fwd(ctypes.byref(p), q, table(*k), table(*v), len(k), chunk_len, block, top_k, index, out, lse, ws, ws_bytes, None)


def bwd(sp, p, q=A, k=(A,), v=(A,), chunk_len=4096, block=64, top_k=4, index=A, out=A, d_out=A, lse=A, dq=A, dtype=0, acc=0, dk=(A,), dv=(A,), ws=A,
        ws_bytes=WS):
    return sp.lib.slimpipe_attn_block_bwd(ctypes.byref(p), q, table(*k), table(*v), len(k), chunk_len, block, top_k, index, out, d_out, lse, dq, dtype, acc,
                                          table(*dk), table(*dv), 1, ws, ws_bytes, None)


def store(sp, p, k=A, v=A, cache=(A, A, A, A)):
    return sp.lib.slimpipe_attn_kv4_store(ctypes.byref(p), k, v, *cache, None)


def load(sp, p, cache=(A, A, A, A), k=A, v=A):
    return sp.lib.slimpipe_attn_kv4_load(ctypes.byref(p), *cache, k, v, None)


def cached(sp, p, q=A, cache=(A, A, A, A), out=A, lse=A, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_fwd_kv4(ctypes.byref(p), q, *cache, out, lse, ws, ws_bytes, None)


CALLS = [means, select, fwd, bwd, store, load, cached]
BLOCK_CALLS = [means, select, fwd, bwd]


@pytest.mark.parametrize("call", CALLS)
def test_what_validate_refuses_every_call_refuses(sp, call):
    for change, code in ((dict(n_kv_heads=3), SHAPE), (dict(head_dim=96), SHAPE), (dict(s_q=0), SHAPE), (dict(scale=float("nan")), SHAPE),
                         (dict(kv_begin=2000, kv_end=1000), RANGE), (dict(kv_end=5000), RANGE), (dict(q_offset=-1), RANGE),
                         (dict(q_offset=2 ** 62), RANGE), (dict(q_stride_s=1023), STRIDE), (dict(kv_stride_h=0), STRIDE)):
        assert call(sp, params(sp, **change)) == code, change
    assert bwd(sp, params(sp, do_stride_s=12)) == STRIDE


def test_block_lengths_and_chunks(sp):
    p = params(sp)
    for call in BLOCK_CALLS:
        for block in (0, -64, 32, 96, 65, 1 << 17):
            assert call(sp, p, block=block) == SHAPE, (call, block)
        assert call(sp, params(sp, kv_capacity=(1 << 36) + 1)) in (SHAPE, RANGE)
        assert call(sp, params(sp, batch=65535, n_q_heads=2, n_kv_heads=2)) == SHAPE
        assert call(sp, params(sp, kv_capacity=1 << 36, kv_end=1 << 36), **({} if call is select else dict(chunk_len=1 << 36))) == SHAPE      # 2^30 blocks
    for call in (means, fwd, bwd):
        pairs = {} if call is means else dict(v=(A, A))
        if call is bwd:
            pairs.update(dk=(A, A), dv=(A, A))
        assert call(sp, p, chunk_len=1000) == RANGE                              # one chunk that does not hold the capacity
        assert call(sp, p, k=(A, A), chunk_len=2000, **pairs) == RANGE
        assert call(sp, p, k=(A, A), chunk_len=2100, **pairs) == SHAPE           # a chunk is a multiple of 256 keys
        assert call(sp, p, k=(A, A), chunk_len=2048, block=320, **pairs) == SHAPE      # and of the block
    assert means(sp, params(sp, kv_begin=65)) == RANGE


def test_top_k_and_row_limits(sp):
    p = params(sp)
    for call in (select, fwd, bwd):
        for top_k in (0, -1, 65):
            assert call(sp, p, top_k=top_k) == SHAPE, top_k
        assert call(sp, params(sp, s_q=1 << 26), top_k=4) == SHAPE                # 2^31 slots of the kv head
        assert call(sp, params(sp, n_kv_heads=8, batch=16, s_q=1 << 20), top_k=1) == SHAPE      # 2^27 rows
        assert call(sp, params(sp, q_stride_h=1 << 33)) == STRIDE                 # offsets in a kv head's rows past 2^35 elements
        assert call(sp, params(sp, q_stride_h=1 << 62)) == STRIDE
    assert bwd(sp, params(sp, do_stride_h=1 << 33)) == STRIDE
    n = ctypes.c_size_t(0)
    for block, top_k in ((32, 4), (64, 0), (64, 65)):
        assert sp.lib.slimpipe_attn_block_workspace_bytes(ctypes.byref(p), block, top_k, 0, ctypes.byref(n)) == SHAPE
    assert sp.lib.slimpipe_attn_block_workspace_bytes(ctypes.byref(p), 64, 4, 0, None) == NULL


def test_null_and_unaligned_pointers(sp):
    p = params(sp)
    for call, names, byte16 in ((means, ["out"], ["out"]), (select, ["q", "m", "index"], ["q", "m"]), (fwd, ["q", "index", "out", "lse"], ["q", "out"]),
                                (bwd, ["q", "index", "out", "d_out", "lse", "dq"], ["q", "out", "d_out", "dq"]), (store, ["k", "v"], ["k", "v"]),
                                (load, ["k", "v"], ["k", "v"]), (cached, ["q", "out", "lse"], ["q", "out"])):
        for n in names:
            assert call(sp, p, **{n: None}) == NULL, (call, n)
            assert call(sp, p, **{n: ODD if n in byte16 else A + 2}) == ALIGN, (call, n)
    for call, names in ((means, ["k"]), (fwd, ["k", "v"]), (bwd, ["k", "v", "dk", "dv"])):
        for n in names:
            assert call(sp, p, **{n: (None,)}) == NULL, (call, n)
            assert call(sp, p, **{n: (ODD,)}) == ALIGN, (call, n)
    for call in (store, load, cached):
        for i in range(4):
            assert call(sp, p, cache=[None if j == i else A for j in range(4)]) == NULL
            if i % 2 == 0:
                assert call(sp, p, cache=[ODD if j == i else A for j in range(4)]) == ALIGN
    assert means(sp, p, k=()) == SHAPE


def test_workspaces(sp):
    def size(f, *args):
        n = ctypes.c_size_t(0)
        assert f(*args, ctypes.byref(n)) == 0
        return n.value
    p = params(sp)
    for is_bwd, call in ((0, fwd), (1, bwd)):
        n = size(sp.lib.slimpipe_attn_block_workspace_bytes, ctypes.byref(p), 64, 4, is_bwd)
        assert n >= 8 * 512 * 4 * 128 * 4
        assert call(sp, p, ws_bytes=n - 1) == WORKSPACE and call(sp, p, ws=None) == WORKSPACE and call(sp, p, ws=ODD) == ALIGN
    token = params(sp, s_q=1, q_offset=4095, kv_end=4096)
    n = size(sp.lib.slimpipe_attn_kv4_workspace_bytes, ctypes.byref(token))
    assert n >= 2 * 8 * 128 * 4                    # a token's keys are cut into ranges
    assert cached(sp, token, ws_bytes=n - 1) == WORKSPACE and cached(sp, token, ws=None) == WORKSPACE and cached(sp, token, ws=ODD) == ALIGN
    assert sp.lib.slimpipe_attn_kv4_workspace_bytes(ctypes.byref(token), None) == NULL
    # a call that fills the GPU has no ranges and needs no workspace
    assert size(sp.lib.slimpipe_attn_kv4_workspace_bytes, ctypes.byref(params(sp, s_q=16384))) == 0


def test_backward_dtypes(sp):
    assert bwd(sp, params(sp), dtype=7) == SHAPE
    assert bwd(sp, params(sp), dtype=sp.BF16, acc=1) == SHAPE


def test_cache_layout_and_limits(sp):
    for call in (store, load, cached):
        assert call(sp, params(sp, kv_stride_s=136)) == STRIDE                   # not whole groups of 32
        assert call(sp, params(sp, kv_stride_b=4096 * 128 + 16)) == STRIDE
        assert call(sp, params(sp, batch=65535, n_q_heads=2, n_kv_heads=2)) == SHAPE
        big = params(sp, kv_capacity=1 << 35, kv_end=1 << 35)
        assert call(sp, big) == SHAPE
    assert store(sp, params(sp, q_offset=4000)) == RANGE                         # rows 4000 .. 4511 of 4096
    assert store(sp, params(sp, q_offset=1 << 40)) == RANGE
    assert cached(sp, params(sp, s_q=1 << 24)) == SHAPE                          # 2^27 rows


def test_binding_refuses_what_does_not_fit_together(sp, monkeypatch):
    """Shapes, dtypes and layouts that the C call cannot see."""
    import torch
    import paper_2504_14519_amd.binding as binding
    monkeypatch.setattr(binding, "_stream", lambda: None)      # (there is no device to ask; every call below is refused before it uses one)
    q, k = torch.zeros(1, 4, 8, 64).bfloat16(), torch.zeros(1, 256, 2, 64).bfloat16()
    index = torch.zeros(1, 8, 4, 2, dtype=torch.int32)
    bad = [index.long(), index[..., :1, :], index.transpose(2, 3), torch.zeros(1, 8, 4, 4, dtype=torch.int32)[..., ::2]]
    for i in bad:
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_fwd(q, k, k, i, 0, 0, 256, 64)
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_workspace_bytes(q, k, i, 0, 0, 256, 64)
    other = torch.zeros(1, 2, 256, 64).bfloat16().transpose(1, 2)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_block_fwd(q, k, other, index, 0, 0, 256, 64)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_block_fwd(q, [k, k], [k], index, 0, 0, 256, 64)
    acc = torch.zeros(1, 256, 2, 64)
    lse = torch.zeros(1, 8, 4)
    for dk, dv, dq in ((acc[:, :128], acc, None), (acc, acc.transpose(1, 2).contiguous().transpose(1, 2), None), (acc, acc, torch.zeros(1, 4, 8, 128)[..., ::2])):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_bwd(q, k, k, index, q, q, lse, 0, 0, 256, 64, dk, dv, dq=dq)
    for m in (torch.zeros(1, 2, 3, 64), torch.zeros(1, 2, 4, 64).double(), torch.zeros(1, 4, 2, 64).transpose(1, 2)):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_means(k, 0, 256, 64, means=m)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_block_select(q, torch.zeros(1, 2, 4, 64), 0, 0, 256, 64, 3, index=index)
    for block, top_k in ((0, 2), (100, 2), (64, 65), (64, 0)):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_select(q, torch.zeros(1, 2, 4, 64), 0, 0, 4 * block, block, top_k)
        if block != 64:
            with pytest.raises(sp.SlimpipeError):
                sp.slimpipe_attn_block_means(k, 0, 256, block)
    cache = sp.KvCache4.empty(1, 300, 2, 64, device="cpu")
    for wrong in (cache._replace(v_codes=cache.v_codes[..., :16]), cache._replace(v_scales=cache.v_scales[:, :200]), cache._replace(k_scales=cache.k_scales.int()),
                  cache._replace(v_scales=cache.v_scales[0]), cache._replace(v_codes=cache.v_codes.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)),
                  cache._replace(k_codes=cache.k_codes[0])):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_kv4_store(k, k, wrong, 0)
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_fwd_kv4(q, wrong, 0, 0, 256)
    for rows, v in ((k[..., :32], k[..., :32]), (k, other), (k[:, :, :1], k[:, :, :1])):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_kv4_store(rows, v, cache, 0)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv4_store(k, k, cache, 100)                             # rows 100 .. 355 of 300
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv4_load(cache, 0, 301)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv4_load(cache, 0, 4, k_rows=k, v_rows=k)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_fwd_kv4(torch.zeros(1, 4, 8, 128).bfloat16(), cache, 0, 0, 256)
