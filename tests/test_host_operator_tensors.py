"""CPU-only: what the wrappers of sparse attention and of the 4-bit cache refuse about the tensors they are given, before the library sees an
address.  The library knows shapes and element widths from its parameters alone: a tensor of another dtype or size would be read or
written as what it is not, or past its end."""
import pytest
import torch

B, S, HQ, H, D, N, L, K = 2, 4, 8, 2, 64, 256, 64, 2
bf16, f32 = torch.bfloat16, torch.float32


class Reached(Exception):
    pass


class Library:
    """The library with its launching entry points taken out: a call that gets there has passed every check of the wrapper."""

    def __init__(self, lib):
        self.lib = lib

    def __getattr__(self, name):
        if name in ("slimpipe_attn_strerror", "slimpipe_attn_block_workspace_bytes", "slimpipe_attn_kv4_workspace_bytes"):
            return getattr(self.lib, name)

        def reached(*args):
            raise Reached(name)
        return reached


@pytest.fixture
def sp(monkeypatch):
    import paper_2504_14519_amd as sp_
    import paper_2504_14519_amd.binding as binding
    monkeypatch.setattr(binding, "lib", Library(binding.lib))
    monkeypatch.setattr(binding, "_stream", lambda: None)
    return sp_


def t(*shape, dtype=bf16):
    return torch.zeros(shape, dtype=dtype)


def right(sp):
    """Tensors that fit together, by argument name."""
    return dict(q=t(B, S, HQ, D), k=t(B, N, H, D), v=t(B, N, H, D), out=t(B, S, HQ, D), d_out=t(B, S, HQ, D), lse=t(B, HQ, S, dtype=f32),
                index=t(B, HQ, S, K, dtype=torch.int32), dq=t(B, S, HQ, D), dk=t(B, N, H, D, dtype=f32), dv=t(B, N, H, D, dtype=f32),
                means=t(B, H, N // L, D, dtype=f32), cache=sp.KvCache4.empty(B, N, H, D, device="cpu"), k_rows=t(B, S, H, D), v_rows=t(B, S, H, D),
                ws=t(1 << 22, dtype=torch.uint8), dtype=sp.BF16)


CALLS = {
    "means": lambda sp, a: sp.slimpipe_attn_block_means(a["k"], 0, N, L, means=a["means"]),
    "select": lambda sp, a: sp.slimpipe_attn_block_select(a["q"], a["means"], 0, 0, N, L, K, index=a["index"]),
    "fwd": lambda sp, a: sp.slimpipe_attn_block_fwd(a["q"], a["k"], a["v"], a["index"], 0, 0, N, L, out_dtype=a["dtype"], out=a["out"], lse=a["lse"],
                                                    workspace=a["ws"]),
    "bwd": lambda sp, a: sp.slimpipe_attn_block_bwd(a["q"], a["k"], a["v"], a["index"], a["out"], a["d_out"], a["lse"], 0, 0, N, L, a["dk"], a["dv"],
                                                    dq=a["dq"], dq_dtype=a["dtype"], workspace=a["ws"]),
    "store": lambda sp, a: sp.slimpipe_attn_kv4_store(a["k_rows"], a["v_rows"], a["cache"], 0),
    "load": lambda sp, a: sp.slimpipe_attn_kv4_load(a["cache"], 0, S, k_rows=a["k_rows"], v_rows=a["v_rows"]),
    "fwd_kv4": lambda sp, a: sp.slimpipe_attn_fwd_kv4(a["q"], a["cache"], 0, 0, N, out_dtype=a["dtype"], out=a["out"], lse=a["lse"], workspace=a["ws"]),
}


def refuses(sp, call, **change):
    with pytest.raises(sp.SlimpipeError):
        CALLS[call](sp, {**right(sp), **change})


def accepts(sp, call, **change):
    with pytest.raises(Reached):
        CALLS[call](sp, {**right(sp), **change})


@pytest.mark.parametrize("call", list(CALLS))
def test_tensors_that_fit_reach_the_library(sp, call):
    accepts(sp, call)


@pytest.mark.parametrize("call,names", [("means", "k"), ("select", "q"), ("fwd", "q k v"), ("bwd", "q k v out d_out"), ("store", "k_rows v_rows"),
                                        ("load", "k_rows v_rows"), ("fwd_kv4", "q")])
def test_dtypes_of_bf16_tensors(sp, call, names):
    for name in names.split():
        shape = right(sp)[name].shape
        for dtype in (f32, torch.float16, torch.int16):
            refuses(sp, call, **{name: t(*shape, dtype=dtype)})
    if "k_rows" in names:                                     # both wrong in the same way
        refuses(sp, call, k_rows=t(B, S, H, D, dtype=torch.float16), v_rows=t(B, S, H, D, dtype=torch.float16))
    if call in ("fwd", "bwd"):
        refuses(sp, call, k=t(B, N, H, D, dtype=f32), v=t(B, N, H, D, dtype=f32))


@pytest.mark.parametrize("call,names", [("fwd", "lse"), ("bwd", "lse dk dv"), ("fwd_kv4", "lse")])
def test_dtypes_of_float32_tensors(sp, call, names):
    for name in names.split():
        shape = right(sp)[name].shape
        for dtype in (bf16, torch.float64, torch.float16):
            refuses(sp, call, **{name: t(*shape, dtype=dtype)})


@pytest.mark.parametrize("call,name", [("fwd", "out"), ("fwd_kv4", "out"), ("bwd", "dq")])
def test_a_result_has_the_dtype_that_the_call_names(sp, call, name):
    shape = right(sp)[name].shape
    accepts(sp, call, dtype=sp.F32, **{name: t(*shape, dtype=f32)})
    refuses(sp, call, dtype=sp.F32, **{name: t(*shape)})                # float32 stores would run past its end
    refuses(sp, call, dtype=sp.BF16, **{name: t(*shape, dtype=f32)})
    refuses(sp, call, dtype=sp.BF16, **{name: t(*shape, dtype=torch.float16)})


# A right tensor's place may be taken by one of these: another batch, fewer rows, other heads, another head_dim, one dimension less, elements that
# do not follow each other.
def misfits(x):
    wide = torch.zeros(x.shape[:-1] + (2 * x.shape[-1],), dtype=x.dtype)
    return [x[:1].clone(), x[:, :x.shape[1] - 1].clone(), x[:, :, :1].clone(), wide, wide[..., ::2], x[0]]


@pytest.mark.parametrize("call,names", [("means", "means"), ("select", "q means index"), ("fwd", "q index out"), ("bwd", "q index out d_out dq"),
                                        ("load", "k_rows v_rows"), ("fwd_kv4", "out")])
def test_shapes(sp, call, names):
    for name in names.split():
        for i, x in enumerate(misfits(right(sp)[name])):
            # (an index of more slots, and means of fewer heads or blocks, are those of another call)
            if not (name == "index" and call != "select" and i == 3) and not (name == "means" and call == "select" and i in (1, 2)):
                refuses(sp, call, **{name: x})


@pytest.mark.parametrize("call,names", [("fwd", "k v"), ("bwd", "k v dk dv")])
def test_shapes_of_keys(sp, call, names):
    for name in names.split():
        for x in misfits(right(sp)[name]):
            refuses(sp, call, **{name: x})
    for x in misfits(right(sp)["k"])[:1] + misfits(right(sp)["k"])[3:]:      # all of them alike, and none fits q
        refuses(sp, call, k=x, v=x, dk=x.float(), dv=x.float())


@pytest.mark.parametrize("call", ["means", "fwd", "bwd"])
def test_chunk_lists(sp, call):
    a = right(sp)
    change = {n: [a[n], a[n]] for n in ("k", "v", "dk", "dv")}
    change["means"] = t(B, H, 2 * N // L, D, dtype=f32)
    accepts(sp, call, **change)
    for name in {"means": "k", "fwd": "k v", "bwd": "k v dk dv"}[call].split():
        for x in misfits(a[name]):
            refuses(sp, call, **{**change, name: [a[name], x]})
        refuses(sp, call, **{**change, name: []})
    refuses(sp, call, **{**change, "k": [], "v": [], "dk": [], "dv": []})


@pytest.mark.parametrize("call", ["means", "select", "fwd_kv4"])
def test_shapes_without_a_partner(sp, call):
    """What has nothing of its own size beside it: elements that do not follow each other, dimensions that are missing."""
    name = "k" if call == "means" else "q"
    x = right(sp)[name]
    for wrong in (torch.zeros(x.shape[:-1] + (2 * D,), dtype=bf16)[..., ::2], x[0]):
        refuses(sp, call, **{name: wrong})
    refuses(sp, call, **{name: t(*x.shape[:-1], 2 * D)})
    if call == "fwd_kv4":
        refuses(sp, call, q=x[:1].clone(), out=x[:1].clone(), lse=t(1, HQ, S, dtype=f32))


@pytest.mark.parametrize("call", ["fwd", "bwd", "fwd_kv4"])
def test_lse_is_contiguous_and_has_the_rows(sp, call):
    for x in (t(B, S, HQ, dtype=f32).transpose(1, 2), t(B, HQ, S - 1, dtype=f32), t(B, HQ - 1, S, dtype=f32), t(1, HQ, S, dtype=f32), t(B, HQ * S, dtype=f32),
              t(B, HQ, 2 * S, dtype=f32)[..., ::2], t(B, HQ, 1, dtype=f32).expand(B, HQ, S)):
        refuses(sp, call, lse=x)
    accepts(sp, call, lse=t(2 * B * HQ * S, dtype=f32)[B * HQ * S:].view(B, HQ, S))      # a part of a larger one


@pytest.mark.parametrize("call", ["store", "load"])
def test_cache_rows(sp, call):
    wide = torch.zeros((B, S, H, 2 * D), dtype=bf16)[..., ::2]
    refuses(sp, call, k_rows=wide, v_rows=wide)
    for x in misfits(right(sp)["k_rows"]):
        if call == "load" or x.shape[1:] != (S - 1, H, D):
            refuses(sp, call, k_rows=x, v_rows=x)
    packed = t(B, S, 3 * H, D)
    accepts(sp, call, k_rows=packed[:, :, :H], v_rows=packed[:, :, H:2 * H])             # heads of a packed projection


def test_load_of_a_range_that_ends_before_it_begins(sp):
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv4_load(right(sp)["cache"], 5, 4)


@pytest.mark.parametrize("call", ["fwd", "bwd", "fwd_kv4"])
def test_a_workspace_is_one_piece(sp, call):
    refuses(sp, call, ws=t(1, dtype=torch.uint8).expand(1 << 22))


def test_workspace_queries(sp):
    a = right(sp)
    for x in (t(1, N, H, D), t(B, N, H, 2 * D), t(N, H, D)):
        with pytest.raises(sp.SlimpipeError):
            sp.slimpipe_attn_block_workspace_bytes(a["q"], x, a["index"], 0, 0, N, L)
    with pytest.raises(sp.SlimpipeError):
        sp.slimpipe_attn_kv4_workspace_bytes(a["q"][0], a["cache"], 0, 0, N)


@pytest.mark.parametrize("call", list(CALLS))
def test_tensors_of_another_device(sp, monkeypatch, call):
    """Every tensor has to be on the current device, whose stream the kernels run on; here that is said to be a GPU, and the tensors are not there."""
    import paper_2504_14519_amd.binding as binding
    monkeypatch.setattr(binding, "_current_device", lambda: 0, raising=False)
    refuses(sp, call)


def test_current_device_of_this_host(sp):
    import paper_2504_14519_amd.binding as binding
    if torch.cuda.device_count() == 0:
        assert binding._current_device() == -1 == t(1).get_device()


@pytest.mark.parametrize("name", ["k_rows", "v_rows"])
def test_load_allocates_one_of_two(sp, name):
    """The other one has gaps: a part of a packed tensor."""
    for given in (t(B, S, H, D), t(B, S, 3 * H, D)[:, :, H:2 * H], t(B, H, S, D).transpose(1, 2), t(B, S + 3, H, D)[:, :S]):
        accepts(sp, "load", k_rows=None, v_rows=None)
        accepts(sp, "load", **{"k_rows": None, "v_rows": None, name: given})


def test_workspace_queries_look_at_sizes_alone(sp):
    """Nothing is read: stand-ins of another dtype, or without memory, will do."""
    a = right(sp)
    want = sp.slimpipe_attn_block_workspace_bytes(a["q"], a["k"], a["index"], 0, 0, N, L)
    for how in (dict(dtype=f32), dict(device="meta")):
        q, k = (torch.empty(a[n].shape, **{"dtype": bf16, **how}) for n in "qk")
        index = torch.empty(a["index"].shape, dtype=torch.int32, device=q.device)
        assert sp.slimpipe_attn_block_workspace_bytes(q, k, index, 0, 0, N, L) == want
        assert sp.slimpipe_attn_block_workspace_bytes(q, [k, k], index, 0, 0, N, L, True, True) > 0
        assert sp.slimpipe_attn_kv4_workspace_bytes(q, a["cache"], 0, 0, N) == sp.slimpipe_attn_kv4_workspace_bytes(a["q"], a["cache"], 0, 0, N)
