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
