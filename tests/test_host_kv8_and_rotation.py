"""CPU-only checks of the 8-bit cache, of eviction from it and of the norm and rotation of queries and keys at the boundary: what is refused, with which code,
before anything touches a device; what the wrappers refuse about tensors; workspace sizes; the definition that the GPU tests go by."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_util as ku

NULL, SHAPE, RANGE, STRIDE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5, -6
A, ODD, FAR = 0x1000, 0x1008, 1 << 44            # addresses that are never read: a call is refused first
WS = 1 << 50


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


def ref(p):
    return ctypes.byref(p) if p is not None else None


def store(sp, p, block=64, k=A, v=A, cache=(A, A, A, A)):
    return sp.lib.slimpipe_attn_kv8_store(ref(p), block, k, v, *cache, None)


def load(sp, p, block=64, cache=(A, A, A, A), k=A, v=A):
    return sp.lib.slimpipe_attn_kv8_load(ref(p), block, *cache, k, v, None)


def cached(sp, p, block=64, q=A, cache=(A, A, A, A), out=A, lse=A, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_fwd_kv8(ref(p), block, q, *cache, out, lse, ws, ws_bytes, None)


def weights(sp, p, block=64, q=A, k=(A, A), lse=A, previous=None, decay=1.0, out=A, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_kv8_weights(ref(p), block, q, *k, lse, previous, decay, out, ws, ws_bytes, None)


def gather(sp, p, block=64, index=A, keep=10, cache=(A, A, A, A), w=None, to=None, to_cache=(FAR, FAR + (1 << 30), FAR + (1 << 31), FAR + (1 << 32)), kept=None):
    return sp.lib.slimpipe_attn_kv8_gather(ref(p), block, index, keep, *cache, w, ref(to or p), *to_cache, kept, None)


def keep(sp, w=A, planes=4, capacity=1000, rows=900, kept=100, recent=10, index=A, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_kv8_keep(w, planes, capacity, rows, kept, recent, index, ws, ws_bytes, None)


CALLS = [store, load, cached, weights, gather]


@pytest.mark.parametrize("call", CALLS)
def test_what_every_call_on_the_cache_refuses(sp, call):
    for change, code in ((dict(n_kv_heads=3), SHAPE), (dict(head_dim=96), SHAPE), (dict(s_q=0), SHAPE), (dict(scale=float("nan")), SHAPE),
                         (dict(kv_begin=2000, kv_end=1000), RANGE), (dict(kv_end=5000), RANGE), (dict(q_offset=-1), RANGE),
                         (dict(q_offset=2 ** 62), RANGE), (dict(q_stride_s=1023), STRIDE), (dict(kv_stride_h=0), STRIDE),
                         (dict(kv_stride_s=136), STRIDE), (dict(kv_stride_b=4096 * 128 + 8), STRIDE),      # whole pieces of 16 bytes
                         (dict(kv_capacity=(1 << 36) + 1), SHAPE), (dict(batch=65535, n_q_heads=2, n_kv_heads=2), SHAPE),
                         (dict(n_kv_heads=8, batch=16, s_q=1 << 20), SHAPE), (dict(kv_capacity=1 << 31, kv_end=(1 << 30) + 1), SHAPE)):
        assert call(sp, params(sp, **change)) == code, change
    for block in (0, -64, 8, 48, 63, 512, 1 << 20):
        assert call(sp, params(sp), block=block) == SHAPE, block
    assert call(sp, None) == NULL


def test_pointers(sp):
    p = params(sp)
    for i in range(4):
        hole = tuple(None if j == i else A for j in range(4))
        crooked = tuple(A + 8 if j == i else A for j in range(4))
        for call in (store, load, cached):
            assert call(sp, p, cache=hole) == NULL
            if i % 2 == 0:
                assert call(sp, p, cache=crooked) == ALIGN
        assert gather(sp, p, cache=hole) == NULL and gather(sp, p, to_cache=hole) == NULL
    for call, name in ((store, "k"), (store, "v"), (load, "k"), (load, "v"), (cached, "q"), (cached, "out"), (cached, "lse"), (weights, "q"), (weights, "lse"),
                       (weights, "out"), (gather, "index")):
        assert call(sp, p, **{name: None}) == NULL, (call, name)
        assert call(sp, p, **{name: 0x1002}) == ALIGN, (call, name)
    assert weights(sp, p, k=(None, A)) == NULL and weights(sp, p, k=(A, None)) == NULL and weights(sp, p, k=(ODD, A)) == ALIGN
    assert weights(sp, p, previous=0x1002) == ALIGN
    assert weights(sp, p, decay=float("nan")) == SHAPE and weights(sp, p, decay=float("inf")) == SHAPE


def test_ranges_of_stores_and_moves(sp):
    assert store(sp, params(sp, q_offset=4096 - 511)) == RANGE
    p = params(sp)
    assert gather(sp, p, keep=-1) == RANGE and gather(sp, p, keep=4097) == RANGE
    assert gather(sp, p, to=params(sp, kv_capacity=9, kv_end=9)) == RANGE
    for change in (dict(batch=2), dict(n_kv_heads=2), dict(head_dim=64)):
        assert gather(sp, p, to=params(sp, **change)) == SHAPE
    assert gather(sp, p, w=A) == NULL and gather(sp, p, kept=A) == NULL
    # the caches, and the sums, may not share memory: codes of the one in codes or scales of the other, sums in sums
    there = A + 4096 * 128
    assert gather(sp, p, to_cache=(A, FAR, FAR, FAR)) == RANGE
    assert gather(sp, p, to_cache=(there - 16, FAR, FAR, FAR)) == RANGE
    assert gather(sp, p, to_cache=(FAR, A + 100, FAR, FAR)) == RANGE
    assert gather(sp, p, w=FAR + (1 << 40), kept=FAR + (1 << 40) + 4 * 4095) == RANGE


def test_keep(sp):
    for change, code in ((dict(w=None), NULL), (dict(index=None), NULL), (dict(planes=0), SHAPE), (dict(planes=65536), SHAPE), (dict(rows=0), SHAPE),
                         (dict(rows=(1 << 30) + 1, capacity=1 << 31), SHAPE), (dict(rows=1001), RANGE), (dict(kept=0), RANGE), (dict(kept=901), RANGE),
                         (dict(recent=-1), RANGE), (dict(recent=101), RANGE), (dict(w=0x1001), ALIGN), (dict(index=0x1002), ALIGN),
                         (dict(rows=40000, capacity=40000, ws=None), WORKSPACE), (dict(rows=40000, capacity=40000, ws_bytes=1000), WORKSPACE),
                         (dict(rows=40000, capacity=40000, ws=ODD), ALIGN)):
        assert keep(sp, **change) == code, change
    n = ctypes.c_size_t(7)
    assert sp.lib.slimpipe_attn_kv8_keep_workspace_bytes(4, 16384, 100, ctypes.byref(n)) == 0 and n.value == 0
    assert sp.lib.slimpipe_attn_kv8_keep_workspace_bytes(4, 16385, 100, ctypes.byref(n)) == 0 and n.value > 0
    assert sp.lib.slimpipe_attn_kv8_keep_workspace_bytes(4, 100, 101, ctypes.byref(n)) == RANGE
    assert sp.lib.slimpipe_attn_kv8_keep_workspace_bytes(4, 100, 50, None) == NULL


def test_workspaces(sp):
    n = ctypes.c_size_t(0)
    size = lambda f, p: (f(ref(p), 64, ctypes.byref(n)), n.value)[1]
    fwd, sums = sp.lib.slimpipe_attn_kv8_workspace_bytes, sp.lib.slimpipe_attn_kv8_weights_workspace_bytes
    slice_ = params(sp)                                       # 4096 rows of a kv head: room for a copy of 1536 keys and values
    assert size(fwd, slice_) >= 2 * 1536 * 128 * 2
    # a piece of which early rows see nothing is converted tile by tile: no copy, the results of its ranges of 128 keys or more
    assert size(fwd, params(sp, kv_begin=1025)) <= 511 // 128 * 512 * 8 * 129 * 4
    early = params(sp, s_q=3000, kv_begin=1025, kv_end=4024)
    need = size(fwd, early)
    assert need > 0 and cached(sp, early, ws=None) == WORKSPACE and cached(sp, early, ws_bytes=need - 1) == WORKSPACE
    token = params(sp, s_q=1, q_offset=4095, kv_end=4096)
    need = size(fwd, token)
    assert 0 < need < 1 << 20 and size(fwd, params(sp, s_q=1, q_offset=100, kv_end=101)) == 0
    assert cached(sp, token, ws=None) == WORKSPACE and cached(sp, token, ws_bytes=need - 1) == WORKSPACE and cached(sp, token, ws=ODD) == ALIGN
    assert size(sums, token) == 0
    need = size(sums, slice_)
    assert need > 0
    assert weights(sp, slice_, ws=None) == WORKSPACE and weights(sp, slice_, ws_bytes=need - 1) == WORKSPACE and weights(sp, slice_, ws=ODD) == ALIGN
    for f in (fwd, sums):
        assert f(ref(slice_), 64, None) == NULL and f(ref(slice_), 60, ctypes.byref(n)) == SHAPE and f(ref(params(sp, s_q=0)), 64, ctypes.byref(n)) == SHAPE


# ------------------------------------------------------------------------------------------ norm and rotation

def rotation(sp, **change):
    p = sp.RotateParams()
    p.batch, p.rows, p.n_q_heads, p.n_kv_heads, p.head_dim, p.rotate_dim, p.interleaved, p.eps, p.position = 2, 100, 8, 2, 128, 64, 0, 1e-6, 5
    for side, heads in (("q", 8), ("k", 2), ("qo", 8), ("ko", 2)):
        for dim, v in (("b", 100 * heads * 128), ("s", heads * 128), ("h", 128)):
            setattr(p, "%s_stride_%s" % (side, dim), v)
    for k, v in change.items():
        setattr(p, k, v)
    return p


def turn(sp, p, q=A, k=A, wq=A, wk=A, f=A, at=None, qo=A, ko=A):
    return sp.lib.slimpipe_attn_norm_rotate(ref(p), q, k, wq, wk, f, at, qo, ko, None)


def turn_back(sp, p, q=A, k=A, wq=A, wk=A, f=A, at=None, dqo=A, tq=0, dko=A, tk=1, dq=A, dk=A, dwq=A, dwk=A, acc=0, ws=A, ws_bytes=WS):
    return sp.lib.slimpipe_attn_norm_rotate_bwd(ref(p), q, k, wq, wk, f, at, dqo, tq, dko, tk, dq, dk, dwq, dwk, acc, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [turn, turn_back])
def test_norm_rotate_refuses(sp, call):
    assert call(sp, None) == NULL
    for change, code in ((dict(batch=0), SHAPE), (dict(rows=0), SHAPE), (dict(n_q_heads=-1), SHAPE), (dict(n_q_heads=0, n_kv_heads=0), SHAPE),
                         (dict(n_q_heads=65536), SHAPE), (dict(head_dim=96), SHAPE), (dict(rotate_dim=8), SHAPE), (dict(rotate_dim=144), SHAPE),
                         (dict(rotate_dim=-16), SHAPE), (dict(eps=0.0), SHAPE), (dict(eps=1e-40), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
                         (dict(batch=1 << 16, rows=1 << 15), SHAPE), (dict(batch=1 << 14, rows=1 << 14), SHAPE),
                         (dict(batch=1, rows=(1 << 28) // 10 + 1), SHAPE), (dict(batch=1, rows=1 << 28, n_q_heads=1, n_kv_heads=0), SHAPE), (dict(position=-1), RANGE),
                         (dict(position=(1 << 52) - 99), RANGE), (dict(q_stride_s=4), STRIDE), (dict(ko_stride_h=64), STRIDE), (dict(qo_stride_b=0), STRIDE),
                         (dict(k_stride_h=-128), STRIDE)):
        assert call(sp, rotation(sp, **change)) == code, change
    p = rotation(sp)
    for name in ("q", "k", "f"):
        assert call(sp, p, **{name: None}) == NULL, name
    for name, at in (("q", ODD), ("k", ODD), ("wq", 0x1002), ("wk", 0x1001), ("f", 0x1004), ("at", 0x1004)):
        assert call(sp, p, **{name: at}) == ALIGN, name


def test_norm_rotate_results(sp):
    p = rotation(sp)
    assert turn(sp, p, qo=None) == NULL and turn(sp, p, ko=None) == NULL and turn(sp, p, qo=ODD) == ALIGN and turn(sp, p, ko=ODD) == ALIGN
    for name in ("dqo", "dko", "dq", "dk"):
        assert turn_back(sp, p, **{name: None}) == NULL and turn_back(sp, p, **{name: ODD}) == ALIGN, name
    assert turn_back(sp, p, tq=2) == SHAPE and turn_back(sp, p, tk=-1) == SHAPE
    assert turn_back(sp, p, wq=None) == NULL and turn_back(sp, p, wk=None) == NULL       # a gradient of no weight
    n = ctypes.c_size_t(0)
    assert sp.lib.slimpipe_attn_norm_rotate_workspace_bytes(ref(p), ctypes.byref(n)) == 0 and n.value > 0
    assert turn_back(sp, p, ws=None) == WORKSPACE and turn_back(sp, p, ws_bytes=n.value - 1) == WORKSPACE and turn_back(sp, p, ws=ODD) == ALIGN
    assert sp.lib.slimpipe_attn_norm_rotate_workspace_bytes(ref(p), None) == NULL
    assert sp.lib.slimpipe_attn_norm_rotate_workspace_bytes(None, ctypes.byref(n)) == NULL


# ------------------------------------------------------------------------------------------ tensors

B, S, HQ, H, D, N, L, KEEP = 2, 4, 8, 2, 64, 96, 32, 20
bf16, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Reached(Exception):
    pass


class Library:
    """The library with its launching entry points taken out: a call that gets there has passed every check of the wrapper."""

    def __init__(self, lib):
        self.lib = lib

    def __getattr__(self, name):
        if name == "slimpipe_attn_strerror" or name.endswith("workspace_bytes"):
            return getattr(self.lib, name)

        def reached(*args):
            raise Reached(name)
        return reached


@pytest.fixture
def wrapped(sp, monkeypatch):
    import paper_2504_14519_amd.binding as binding
    monkeypatch.setattr(binding, "lib", Library(binding.lib))
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return sp


def t(*shape, dtype=bf16):
    return torch.zeros(shape, dtype=dtype)


def right():
    """Tensors that fit together, by argument name."""
    return dict(q=t(B, S, HQ, D), k=t(B, S, H, D), v=t(B, S, H, D), out=t(B, S, HQ, D), lse=t(B, HQ, S, dtype=f32), q_out=t(B, S, HQ, D), k_out=t(B, S, H, D),
                dq_out=t(B, S, HQ, D), dk_out=t(B, S, H, D, dtype=f32), dq=t(B, S, HQ, D), dk=t(B, S, H, D), wq=t(D, dtype=f32), wk=t(D, dtype=f32),
                dwq=t(D, dtype=f32), dwk=t(D, dtype=f32), f=t(D // 2, dtype=torch.float64), at=t(B, S, dtype=torch.int64), sums=t(B, H, N, dtype=f32),
                before=t(B, H, N, dtype=f32), index=t(B, H, KEEP, dtype=i32), kept_sums=t(B, H, 40, dtype=f32), ws=t(1 << 20, dtype=u8),
                kc=t(B, N, H, D, dtype=u8), ks=t(B, 3, H, dtype=u8), vc=t(B, N, H, D, dtype=u8), vs=t(B, 3, H, dtype=u8),
                kc2=t(B, 40, H, D, dtype=u8), ks2=t(B, 2, H, dtype=u8), vc2=t(B, 40, H, D, dtype=u8), vs2=t(B, 2, H, dtype=u8))


def one(sp, a):
    return sp.KvCache8(a["kc"], a["ks"], a["vc"], a["vs"], L)


def two(sp, a):
    return sp.KvCache8(a["kc2"], a["ks2"], a["vc2"], a["vs2"], L)


CACHE = " kc ks vc vs"
WRAPPED = [
    ("q k wq wk f at q_out k_out", lambda sp, a: sp.slimpipe_attn_norm_rotate(a["q"], a["k"], a["wq"], a["wk"], a["f"], a["at"], q_out=a["q_out"], k_out=a["k_out"])),
    ("q k wq wk f at dq_out dk_out dq dk dwq dwk ws",
     lambda sp, a: sp.slimpipe_attn_norm_rotate_bwd(a["q"], a["k"], a["wq"], a["wk"], a["f"], a["at"], a["dq_out"], a["dk_out"], dq=a["dq"], dk=a["dk"],
                                                    dq_weight=a["dwq"], dk_weight=a["dwk"], workspace=a["ws"])),
    ("k v" + CACHE, lambda sp, a: sp.slimpipe_attn_kv8_store(a["k"], a["v"], one(sp, a), 0)),
    ("k v" + CACHE, lambda sp, a: sp.slimpipe_attn_kv8_load(one(sp, a), 0, S, k_rows=a["k"], v_rows=a["v"])),
    ("q out lse" + CACHE, lambda sp, a: sp.slimpipe_attn_fwd_kv8(a["q"], one(sp, a), 0, 0, N, out=a["out"], lse=a["lse"], workspace=a["ws"])),
    ("q lse sums before kc ks", lambda sp, a: sp.slimpipe_attn_kv8_weights(a["q"], one(sp, a), a["lse"], 0, 0, N, weights=a["sums"], previous=a["before"],
                                                                          workspace=a["ws"])),
    ("sums index", lambda sp, a: sp.slimpipe_attn_kv8_keep(a["sums"], N, KEEP, index=a["index"], workspace=a["ws"])),
    ("index sums kept_sums kc2 ks2 vc2 vs2" + CACHE, lambda sp, a: sp.slimpipe_attn_kv8_gather(one(sp, a), a["index"], two(sp, a), a["sums"], a["kept_sums"])),
]
OTHER = {bf16: f32, f32: torch.float64, torch.float64: f32, torch.int64: i32, i32: torch.int64, u8: i32}


@pytest.mark.parametrize("i", range(len(WRAPPED)))
def test_wrappers_refuse_tensors_that_do_not_fit(wrapped, i):
    names, call = WRAPPED[i]
    a = right()
    with pytest.raises(Reached):
        call(wrapped, a)
    for name in names.split():
        x = a[name]
        bad = [x.to(OTHER[x.dtype]), x[..., :-1], x.reshape(-1)[:-1], x.unsqueeze(0)]
        if name in ("dq_out", "dk_out"):
            bad[0] = x.to(torch.float16)
        if x.dim() > 1:
            bad += [torch.cat((x, x), 0), torch.cat((x, x), 1).narrow(1, 0, x.shape[1]).transpose(-1, -2).contiguous().transpose(-1, -2)]
        if name == "ws":
            bad = [torch.cat((x, x))[::2]]
        if name == "f":
            bad = [bad[0], bad[3], torch.cat((x, x))[::2]]      # (any number of frequencies is a rotation of its own)
        if name == "sums" and names == "sums index":
            bad = [bad[0], bad[2], bad[3]]
        for y in bad:
            try:
                call(wrapped, {**a, name: y})
            except wrapped.SlimpipeError:
                continue
            except Reached:
                pass
            pytest.fail("%s of %r, %r, %r was taken" % (name, tuple(y.shape), y.stride(), y.dtype))


def test_wrappers_beyond_single_tensors(wrapped):
    sp, a = wrapped, right()
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv8_gather(one(sp, a), a["index"], sp.KvCache8(*two(sp, a)[:4], 64))
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv8_gather(one(sp, a), a["index"], two(sp, a), weights=a["sums"])
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv8_load(one(sp, a), 5, 4)
    for block in (0, -32):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_kv8_store(a["k"], a["v"], sp.KvCache8(*one(sp, a)[:4], block), 0)


def test_wrappers_refuse_numbers_that_no_field_holds(wrapped):
    sp, a = wrapped, right()
    rotated = a["q"], a["k"], a["wq"], a["wk"], a["f"]
    for call in (lambda: sp.slimpipe_attn_norm_rotate(*rotated, 0, eps=1e39), lambda: sp.slimpipe_attn_norm_rotate(*rotated, 1 << 63),
                 lambda: sp.slimpipe_attn_norm_rotate(*rotated, 0.5), lambda: sp.slimpipe_attn_kv8_store(a["k"], a["v"], one(sp, a), 1 << 63),
                 lambda: sp.slimpipe_attn_fwd_kv8(a["q"], one(sp, a), 0, 0, N, scale=1e39),
                 lambda: sp.slimpipe_attn_kv8_weights(a["q"], one(sp, a), a["lse"], 0, -1 << 64, N)):
        with pytest.raises(sp.SlimpipeError):
            call()


def test_a_load_of_no_rows(sp, monkeypatch):
    import paper_2504_14519_amd.binding as binding
    monkeypatch.setattr(binding, "_stream", lambda: None)
    k, v = sp.slimpipe_attn_kv8_load(one(sp, right()), 7, 7)
    assert k.shape == v.shape == (B, 0, H, D)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv8_load(one(sp, right()), N + 1, N + 1)


# ------------------------------------------------------------------------------------------ the definition

def test_format_against_the_library_type():
    """kv8_util against torch's own conversion to the same 8-bit float, on every code and on the middles between them."""
    codes = torch.arange(127, dtype=u8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), ku.levels())
    x = np.concatenate([ku.levels(), (ku.levels()[1:] + ku.levels()[:-1]) / 2, np.random.RandomState(0).rand(1000) * 448])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ku.round_to(x, np.ones_like(x)), want)
    assert ku.unit_of(448.0) == 1.0 and ku.unit_of(448.01) == 2.0 and ku.unit_of(0.0) == 2.0 ** -110 and ku.unit_of(3.0e38) == 2.0 ** 120
