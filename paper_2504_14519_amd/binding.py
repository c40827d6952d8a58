"""ctypes binding of libslimpipe_attn.so: argument marshalling only.

Same entry-point names as the C header.  Tensors are torch tensors on the GPU; torch supplies
device memory and the current stream, every step of the computation runs in the library's kernels.
There is no fallback: if the shared library is missing the import fails.
"""
import collections
import ctypes
import math
import os

# torch before the library: the tensors and streams handed to the library come from torch's HIP runtime, so that runtime has
# to be the one already in the process when the library's dependency on libamdhip64 is resolved (loaded the other
# way round, the library can end up on a second runtime instance that sees no device)
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libslimpipe_attn.so")

BF16, F32 = 0, 1


class SlimpipeError(RuntimeError):
    pass


class AttnParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("s_q", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("kv_capacity", ctypes.c_int64), ("q_offset", ctypes.c_int64), ("kv_begin", ctypes.c_int64),
        ("kv_end", ctypes.c_int64), ("scale", ctypes.c_float), ("out_dtype", ctypes.c_int32),
        ("q_stride_b", ctypes.c_int64), ("q_stride_s", ctypes.c_int64), ("q_stride_h", ctypes.c_int64),
        ("kv_stride_b", ctypes.c_int64), ("kv_stride_s", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64),
        ("o_stride_b", ctypes.c_int64), ("o_stride_s", ctypes.c_int64), ("o_stride_h", ctypes.c_int64),
        ("do_stride_b", ctypes.c_int64), ("do_stride_s", ctypes.c_int64), ("do_stride_h", ctypes.c_int64),
    ]


class BwdPlan(ctypes.Structure):
    _fields_ = [
        ("one_launch", ctypes.c_int32), ("dq_first", ctypes.c_int32), ("dkdv_split", ctypes.c_int32), ("dq_ranges", ctypes.c_int32),
        ("dkdv_items", ctypes.c_int64), ("dq_items", ctypes.c_int64), ("compute_units", ctypes.c_int32), ("dq_by_xcd", ctypes.c_int32),
    ]


class CallPath(ctypes.Structure):
    _fields_ = [("small", ctypes.c_int32), ("ranges", ctypes.c_int32), ("dq_tile_keys", ctypes.c_int32), ("dkdv_tile_rows", ctypes.c_int32)]


class SmallBwdPlan(ctypes.Structure):
    _fields_ = [("small", ctypes.c_int32), ("key_blocks", ctypes.c_int32), ("own_statistics", ctypes.c_int32), ("dq_first", ctypes.c_int32)]


def library_path():
    return _LIB_PATH


def _load():
    if not os.path.exists(_LIB_PATH):
        # nothing built yet: compile the HIP library now (hipcc cross-compiles without a GPU).  There is no
        # fallback path: if that fails, so does the import.
        try:
            from .build import build as _build
            _build()
        except Exception as e:
            raise ImportError("libslimpipe_attn.so is not built and building it failed (%s): run "
                              "`python paper_2504_14519_amd/build.py`" % e)
    L = ctypes.CDLL(_LIB_PATH)
    P = ctypes.POINTER(AttnParams)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    L.slimpipe_attn_init.argtypes = []
    L.slimpipe_attn_init.restype = ctypes.c_int
    L.slimpipe_attn_validate.argtypes = [P, ctypes.c_int]
    L.slimpipe_attn_validate.restype = ctypes.c_int
    L.slimpipe_attn_workspace_bytes.argtypes = [P, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    L.slimpipe_attn_workspace_bytes.restype = ctypes.c_int
    L.slimpipe_attn_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_fwd.restype = ctypes.c_int
    L.slimpipe_attn_bwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, i32, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_bwd.restype = ctypes.c_int
    L.slimpipe_attn_bwd_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, i32, vp]
    L.slimpipe_attn_bwd_noalloc.restype = ctypes.c_int
    L.slimpipe_attn_noalloc_max_rows.argtypes = []
    L.slimpipe_attn_noalloc_max_rows.restype = ctypes.c_int
    pp = ctypes.POINTER(vp)
    L.slimpipe_attn_fwd_chunked.argtypes = [P, vp, pp, pp, i32, i64, vp, vp, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_fwd_chunked.restype = ctypes.c_int
    L.slimpipe_attn_bwd_chunked.argtypes = [P, vp, pp, pp, i32, i64, vp, vp, vp, vp, i32, i32, pp, pp, i32, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_bwd_chunked.restype = ctypes.c_int
    L.slimpipe_attn_fwd_ranges.argtypes = [P, vp, pp, pp, i32, i64, i32, ctypes.POINTER(i64), ctypes.POINTER(i64), vp, vp, vp, vp, vp]
    L.slimpipe_attn_fwd_ranges.restype = ctypes.c_int
    L.slimpipe_attn_merge.argtypes = [i32, ctypes.POINTER(vp), ctypes.POINTER(vp), i32, i32, i32, i32, i32, vp, i32, vp, vp]
    L.slimpipe_attn_merge.restype = ctypes.c_int
    L.slimpipe_attn_finalize_bf16.argtypes = [vp, vp, i64, vp]
    L.slimpipe_attn_finalize_bf16.restype = ctypes.c_int
    szp = ctypes.POINTER(ctypes.c_size_t)
    L.slimpipe_attn_block_means.argtypes = [P, pp, i32, i64, i32, vp, vp]
    L.slimpipe_attn_block_means.restype = ctypes.c_int
    L.slimpipe_attn_block_select.argtypes = [P, vp, vp, i32, i32, vp, vp]
    L.slimpipe_attn_block_select.restype = ctypes.c_int
    L.slimpipe_attn_block_workspace_bytes.argtypes = [P, i32, i32, ctypes.c_int, szp]
    L.slimpipe_attn_block_workspace_bytes.restype = ctypes.c_int
    L.slimpipe_attn_block_fwd.argtypes = [P, vp, pp, pp, i32, i64, i32, i32, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_block_fwd.restype = ctypes.c_int
    L.slimpipe_attn_block_bwd.argtypes = [P, vp, pp, pp, i32, i64, i32, i32, vp, vp, vp, vp, vp, i32, i32, pp, pp, i32, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_block_bwd.restype = ctypes.c_int
    L.slimpipe_attn_kv4_store.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    L.slimpipe_attn_kv4_store.restype = ctypes.c_int
    L.slimpipe_attn_kv4_load.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    L.slimpipe_attn_kv4_load.restype = ctypes.c_int
    L.slimpipe_attn_kv4_workspace_bytes.argtypes = [P, szp]
    L.slimpipe_attn_kv4_workspace_bytes.restype = ctypes.c_int
    L.slimpipe_attn_fwd_kv4.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.slimpipe_attn_fwd_kv4.restype = ctypes.c_int
    L.slimpipe_attn_mfma_rate.argtypes = [ctypes.c_int, vp, ctypes.POINTER(ctypes.c_double), vp]
    L.slimpipe_attn_mfma_rate.restype = ctypes.c_int
    L.slimpipe_attn_dq_atomic_probe.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, i32, vp, ctypes.POINTER(ctypes.c_double), vp]
    L.slimpipe_attn_dq_atomic_probe.restype = ctypes.c_int
    L.slimpipe_attn_xcd_rate.argtypes = [i32, i32, vp, vp, vp, vp]
    L.slimpipe_attn_xcd_rate.restype = ctypes.c_int
    L.slimpipe_attn_profile_enable.argtypes = [ctypes.c_int]
    L.slimpipe_attn_profile_enable.restype = ctypes.c_int
    L.slimpipe_attn_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    L.slimpipe_attn_profile_read.restype = ctypes.c_int
    L.slimpipe_attn_bwd_plan.argtypes = [P, i32, ctypes.c_size_t, ctypes.POINTER(BwdPlan)]
    L.slimpipe_attn_bwd_plan.restype = ctypes.c_int
    L.slimpipe_attn_call_path.argtypes = [P, ctypes.c_int, i32, ctypes.c_size_t, ctypes.POINTER(CallPath)]
    L.slimpipe_attn_call_path.restype = ctypes.c_int
    L.slimpipe_attn_small_bwd_plan.argtypes = [P, i32, ctypes.c_size_t, ctypes.POINTER(SmallBwdPlan)]
    L.slimpipe_attn_small_bwd_plan.restype = ctypes.c_int
    L.slimpipe_attn_strerror.argtypes = [ctypes.c_int]
    L.slimpipe_attn_strerror.restype = ctypes.c_char_p
    return L


lib = _load()


def slimpipe_attn_strerror(code):
    return lib.slimpipe_attn_strerror(int(code)).decode()


def _check(rc, what):
    if rc != 0:
        raise SlimpipeError("%s failed: %d (%s)" % (what, rc, slimpipe_attn_strerror(rc)))


def _stream():
    # the raw handle of the current device's current stream, through two private functions of torch: 0.3 us; the public call
    # builds a stream object, 2.9 us
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _same_strides(a, b):
    """Equal shapes and equal strides on every dimension longer than one."""
    if a.stride() == b.stride() and a.shape == b.shape:
        return True
    return a.shape == b.shape and all(sa == sb for n, sa, sb in zip(a.shape, a.stride(), b.stride()) if n > 1)


def _params(q, k, out_like, d_out, q_offset, kv_begin, kv_end, causal, scale, out_dtype):
    # strides as whole tuples: a question to a tensor is 0.1 us, and every call fills one of these (2.3 -> 1.3 us)
    B, s, Hq, D = q.shape
    k_shape, sq, sk, so, sd = k.shape, q.stride(), k.stride(), out_like.stride(), d_out.stride()
    # in the order of AttnParams
    return AttnParams(B, s, Hq, k_shape[2], D, 1 if causal else 0, k_shape[1], q_offset, kv_begin, kv_end,
                      float(scale) if scale is not None else 1.0 / math.sqrt(D), out_dtype, sq[0], sq[1], sq[2],
                      sk[0], sk[1], sk[2], so[0], so[1], so[2], sd[0], sd[1], sd[2])


class _Layout:
    """Shape and strides of anything that has a shape and answers stride(i)."""
    def __init__(self, x):
        self.shape = x.shape
        self._strides = x.stride(0), x.stride(1), x.stride(2)

    def stride(self):
        return self._strides


def make_params(q, k, out_like, q_offset, kv_begin, kv_end, causal, scale, out_dtype=BF16):
    """Fill the parameter block from shapes/strides.  q [B,s,Hq,D], k [B,Nkv,Hkv,D]; the strides of d_out are those of out."""
    out_like = _Layout(out_like)
    return _params(_Layout(q), _Layout(k), out_like, out_like, q_offset, kv_begin, kv_end, causal, scale, out_dtype)


def slimpipe_attn_init():
    """Prepare the current device for launches (needed once per device before a HIP graph capture)."""
    _check(lib.slimpipe_attn_init(), "slimpipe_attn_init")


def slimpipe_attn_validate(params, is_bwd=False):
    return lib.slimpipe_attn_validate(ctypes.byref(params), 1 if is_bwd else 0)


def slimpipe_attn_workspace_bytes(params, is_bwd):
    n = ctypes.c_size_t(0)
    _check(lib.slimpipe_attn_workspace_bytes(ctypes.byref(params), 1 if is_bwd else 0, ctypes.byref(n)), "workspace_bytes")
    return n.value


def _ws(workspace):
    return (workspace.data_ptr(), workspace.numel()) if workspace is not None else (None, 0)


def _outputs(q_slice, out_dtype, out, lse):
    """out and lse of a forward call, allocated where the caller gave none."""
    B, s, Hq, D = q_slice.shape
    if out is None:
        out = torch.empty((B, s, Hq, D), device=q_slice.device, dtype=torch.float32 if out_dtype == F32 else torch.bfloat16)
    if lse is None:
        lse = torch.empty((B, Hq, s), device=q_slice.device, dtype=torch.float32)
    return out, lse


def slimpipe_attn_fwd(q_slice, k_prefix, v_prefix, q_offset, kv_begin, kv_end, causal=True, scale=None,
                      out_dtype=BF16, out=None, lse=None, workspace=None):
    """-> (out, lse).  out [B,s,Hq,D] (bf16 or fp32), lse [B,Hq,s] fp32.  workspace: uint8 tensor the library may
    use to cut a short slice over a long cache into key ranges (slimpipe_attn_workspace_bytes(p, False))."""
    if out is None or lse is None:
        out, lse = _outputs(q_slice, out_dtype, out, lse)
    p = _params(q_slice, k_prefix, out, out, q_offset, kv_begin, kv_end, causal, scale, out_dtype)
    _check(lib.slimpipe_attn_fwd(ctypes.byref(p), q_slice.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(),
                                 out.data_ptr(), lse.data_ptr(), *_ws(workspace), _stream()), "slimpipe_attn_fwd")
    return out, lse


def slimpipe_attn_bwd(q_slice, k_prefix, v_prefix, out, d_out, lse, q_offset, kv_begin, kv_end, dk_acc, dv_acc,
                      causal=True, scale=None, dq=None, dq_dtype=BF16, dq_accumulate=False, dkv_accumulate=True,
                      workspace=None):
    """-> dq.  dk_acc/dv_acc (fp32, shaped like k_prefix) get rows [kv_begin, kv_end) written or incremented."""
    if dq is None:
        dq = torch.empty_like(q_slice, dtype=torch.float32 if dq_dtype == F32 else torch.bfloat16)
    if not (_same_strides(dq, q_slice) and _same_strides(dk_acc, k_prefix) and _same_strides(dv_acc, k_prefix)):
        raise SlimpipeError("dq must have the strides of q; dk_acc/dv_acc those of k")
    p = _params(q_slice, k_prefix, out, d_out, q_offset, kv_begin, kv_end, causal, scale, BF16)
    if workspace is None:
        workspace = torch.empty(slimpipe_attn_workspace_bytes(p, True), device=q_slice.device, dtype=torch.uint8)
    _check(lib.slimpipe_attn_bwd(ctypes.byref(p), q_slice.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(),
                                 out.data_ptr(), d_out.data_ptr(), lse.data_ptr(), dq.data_ptr(), dq_dtype,
                                 1 if dq_accumulate else 0, dk_acc.data_ptr(), dv_acc.data_ptr(),
                                 1 if dkv_accumulate else 0, workspace.data_ptr(), workspace.numel(), _stream()),
           "slimpipe_attn_bwd")
    return dq


def slimpipe_attn_bwd_noalloc(q_slice, k_prefix, v_prefix, out, d_out, lse, q_offset, kv_begin, kv_end, dq, dk_acc, dv_acc,
                              causal=True, scale=None, dq_accumulate=False, dkv_accumulate=True):
    """slimpipe_attn_bwd without a workspace and without any allocation (the binding allocates nothing either: dq is
    the caller's, float32 or bf16 by its dtype).  -> the status code's check; results in dq, dk_acc, dv_acc."""
    if not (_same_strides(dq, q_slice) and _same_strides(dk_acc, k_prefix) and _same_strides(dv_acc, k_prefix)):
        raise SlimpipeError("dq must have the strides of q; dk_acc/dv_acc those of k")
    p = _params(q_slice, k_prefix, out, d_out, q_offset, kv_begin, kv_end, causal, scale, BF16)
    _check(lib.slimpipe_attn_bwd_noalloc(ctypes.byref(p), q_slice.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(),
                                         out.data_ptr(), d_out.data_ptr(), lse.data_ptr(), dq.data_ptr(),
                                         F32 if dq.dtype == torch.float32 else BF16, 1 if dq_accumulate else 0,
                                         dk_acc.data_ptr(), dv_acc.data_ptr(), 1 if dkv_accumulate else 0, _stream()),
           "slimpipe_attn_bwd_noalloc")
    return dq


def _chunk_table(chunks):
    """list of tensors -> ctypes array of device pointers (all chunks share shape and strides)."""
    c0 = chunks[0]
    for c in chunks[1:]:
        if not _same_strides(c, c0):
            raise SlimpipeError("chunks must share shape and strides")
    return (ctypes.c_void_p * len(chunks))(*[c.data_ptr() for c in chunks])


class _ChunkedKV:
    """What _params needs to know of a chunk list: the shape and strides of the virtual prefix."""
    def __init__(self, chunks):
        c0 = chunks[0]
        self.shape = (c0.shape[0], len(chunks) * c0.shape[1], c0.shape[2], c0.shape[3])
        self._strides = c0.stride()

    def stride(self):
        return self._strides


def slimpipe_attn_fwd_chunked(q_slice, k_chunks, v_chunks, q_offset, kv_begin, kv_end, causal=True, scale=None,
                              out_dtype=BF16, out=None, lse=None, workspace=None):
    """As slimpipe_attn_fwd with K/V given as lists of equally shaped chunks [B, chunk_len, Hkv, D]."""
    if out is None or lse is None:
        out, lse = _outputs(q_slice, out_dtype, out, lse)
    p = _params(q_slice, _ChunkedKV(k_chunks), out, out, q_offset, kv_begin, kv_end, causal, scale, out_dtype)
    _check(lib.slimpipe_attn_fwd_chunked(ctypes.byref(p), q_slice.data_ptr(), _chunk_table(k_chunks), _chunk_table(v_chunks),
                                         len(k_chunks), k_chunks[0].shape[1], out.data_ptr(), lse.data_ptr(), *_ws(workspace),
                                         _stream()),
           "slimpipe_attn_fwd_chunked")
    return out, lse


def slimpipe_attn_fwd_ranges(q_slice, k_chunks, v_chunks, q_offset, ranges, causal=True, scale=None, merged=True,
                             out_dtype=BF16, out=None, lse=None):
    """One launch over several key ranges [(kv_begin, kv_end), ...] of one query slice; k_chunks / v_chunks: a list
    of chunks, or one tensor.  -> (part_out [R,B,s,Hq,D] fp32, part_lse [R,B,Hq,s], out, lse); out and lse are the
    merged result, or None with merged=False."""
    if not isinstance(k_chunks, (list, tuple)):
        k_chunks, v_chunks = [k_chunks], [v_chunks]
    B, s, Hq, D = q_slice.shape
    R = len(ranges)
    part_out = torch.empty((R, B, s, Hq, D), device=q_slice.device, dtype=torch.float32)
    part_lse = torch.empty((R, B, Hq, s), device=q_slice.device, dtype=torch.float32)
    out, lse = _outputs(q_slice, out_dtype, out, lse) if merged else (None, None)
    kv, out_like = _ChunkedKV(k_chunks), out if merged else part_out[0]
    p = _params(q_slice, kv, out_like, out_like, q_offset, 0, kv.shape[1], causal, scale, out_dtype)
    begins = (ctypes.c_int64 * R)(*[int(a) for a, _ in ranges])
    ends = (ctypes.c_int64 * R)(*[int(b) for _, b in ranges])
    _check(lib.slimpipe_attn_fwd_ranges(ctypes.byref(p), q_slice.data_ptr(), _chunk_table(k_chunks), _chunk_table(v_chunks),
                                        len(k_chunks), k_chunks[0].shape[1], R, begins, ends, part_out.data_ptr(), part_lse.data_ptr(),
                                        out.data_ptr() if merged else None, lse.data_ptr() if merged else None, _stream()),
           "slimpipe_attn_fwd_ranges")
    return part_out, part_lse, out, lse


def slimpipe_attn_bwd_chunked(q_slice, k_chunks, v_chunks, out, d_out, lse, q_offset, kv_begin, kv_end, dk_chunks, dv_chunks,
                              causal=True, scale=None, dq=None, dq_dtype=BF16, dq_accumulate=False, dkv_accumulate=True,
                              workspace=None):
    """As slimpipe_attn_bwd with K/V and the fp32 dK/dV accumulators given as lists of chunks."""
    if dq is None:
        dq = torch.empty_like(q_slice, dtype=torch.float32 if dq_dtype == F32 else torch.bfloat16)
    if not _same_strides(dq, q_slice):
        raise SlimpipeError("dq must have the strides of q")
    for c in list(dk_chunks) + list(dv_chunks):
        if not _same_strides(c, k_chunks[0]):
            raise SlimpipeError("dk/dv chunks must have the strides of the k chunks")
    p = _params(q_slice, _ChunkedKV(k_chunks), out, d_out, q_offset, kv_begin, kv_end, causal, scale, BF16)
    if workspace is None:
        workspace = torch.empty(slimpipe_attn_workspace_bytes(p, True), device=q_slice.device, dtype=torch.uint8)
    _check(lib.slimpipe_attn_bwd_chunked(ctypes.byref(p), q_slice.data_ptr(), _chunk_table(k_chunks), _chunk_table(v_chunks),
                                         len(k_chunks), k_chunks[0].shape[1], out.data_ptr(), d_out.data_ptr(), lse.data_ptr(),
                                         dq.data_ptr(), dq_dtype, 1 if dq_accumulate else 0, _chunk_table(dk_chunks),
                                         _chunk_table(dv_chunks), 1 if dkv_accumulate else 0, workspace.data_ptr(),
                                         workspace.numel(), _stream()),
           "slimpipe_attn_bwd_chunked")
    return dq


def slimpipe_attn_merge(outs, lses, out_dtype=BF16, out=None, lse=None):
    """Merge partial (out, lse) pairs over disjoint key sets -> (out, lse)."""
    n = len(outs)
    B, s, Hq, D = outs[0].shape
    part_dtype = F32 if outs[0].dtype == torch.float32 else BF16
    for o in outs:
        if not o.is_contiguous():
            raise SlimpipeError("partial outputs must be contiguous")
    if out is None:
        out = torch.empty((B, s, Hq, D), device=outs[0].device, dtype=torch.float32 if out_dtype == F32 else torch.bfloat16)
    if lse is None:
        lse = torch.empty((B, Hq, s), device=outs[0].device, dtype=torch.float32)
    op = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
    lp = (ctypes.c_void_p * n)(*[l.data_ptr() for l in lses])
    _check(lib.slimpipe_attn_merge(n, op, lp, part_dtype, B, s, Hq, D, out.data_ptr(), out_dtype, lse.data_ptr(), _stream()),
           "slimpipe_attn_merge")
    return out, lse


def slimpipe_attn_finalize_bf16(acc, dst=None):
    if dst is None:
        dst = torch.empty(acc.shape, device=acc.device, dtype=torch.bfloat16)
    _check(lib.slimpipe_attn_finalize_bf16(acc.data_ptr(), dst.data_ptr(), acc.numel(), _stream()), "finalize_bf16")
    return dst


def _as_chunks(x):
    return x if isinstance(x, (list, tuple)) else [x]


def _kv_like(chunks):
    return chunks[0] if len(chunks) == 1 else _ChunkedKV(chunks)


# The library takes element widths from its entry points and dtype codes, and extents from q_slice, the keys and the key range alone.  A tensor
# of another dtype would be read or written as what it is not, a narrower or smaller one past its end.  (Few questions to a tensor, each
# asked once: these checks take 0.5 to 2 us of a call.)
_TORCH_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


def _check_rows(name, x, shape, dtype=torch.bfloat16):
    if x.dtype is not dtype or x.shape != shape or len(shape) != 4 or x.stride(3) != 1:
        raise SlimpipeError("%s must be %s, [batch, rows, heads, head_dim] of the call's sizes, head_dim contiguous" % (name, dtype))


def _check_lse(lse, shape):
    if lse.dtype is not torch.float32 or lse.shape != (shape[0], shape[2], shape[1]) or not lse.is_contiguous():
        raise SlimpipeError("lse must be contiguous and float32, [batch, query heads, rows]")


def _check_keys(chunks, q_shape=None, dtype=torch.bfloat16):
    """One tensor or a list of chunks, whose shapes and strides _chunk_table compares."""
    for c in chunks:
        if c.dtype is not dtype:
            raise SlimpipeError("keys and values must be torch.bfloat16, their gradients torch.float32")
    shape = chunks[0].shape if chunks else ()
    if len(shape) != 4 or chunks[0].stride(3) != 1:
        raise SlimpipeError("keys must be [batch, keys, kv heads, head_dim], head_dim contiguous, or a list of such chunks")
    if q_shape is not None and (shape[0] != q_shape[0] or shape[3] != q_shape[3]):
        raise SlimpipeError("q_slice and the keys must have the same batch and head_dim")


_gpus = None


def _current_device():
    """Index of the current GPU; -1, the index of tensors in host memory, where there is none (a call then ends in the library's own checks)."""
    global _gpus
    if _gpus is None:
        _gpus = torch.cuda.device_count()
    return torch._C._cuda_getDevice() if _gpus else -1


def _check_device(*tensors):
    """The kernels run on the current device's current stream: every tensor has to be there."""
    here = _current_device()
    for x in tensors:
        if x.get_device() != here:
            raise SlimpipeError("every tensor of a call must be on the current device")


def _check_workspace(workspace):
    if not workspace.is_contiguous():
        raise SlimpipeError("a workspace must be contiguous")


def _check_index(index, q_shape):
    shape = index.shape
    if (index.dtype is not torch.int32 or len(shape) != 4 or shape[0] != q_shape[0] or shape[1] != q_shape[2] or shape[2] != q_shape[1]
            or not index.is_contiguous()):
        raise SlimpipeError("index must be a contiguous int32 tensor [batch, query heads, rows, top_k]")
    return shape[3]


def _check_means(means, batch, kv_heads, blocks, head_dim):
    if means.dtype != torch.float32 or tuple(means.shape) != (batch, kv_heads, blocks, head_dim) or not means.is_contiguous():
        raise SlimpipeError("means must be a contiguous float32 tensor [batch, kv heads, ceil(keys / block_len), head_dim]")


def slimpipe_attn_block_means(k_chunks, kv_begin, kv_end, block_len, means=None):
    """-> means [B, Hkv, ceil(keys / block_len), D] fp32: those of the blocks that hold a key of [kv_begin, kv_end) are written (kv_begin a
    multiple of block_len), the others left as they are (zero where the call allocates).  k_chunks: one tensor or a list of chunks."""
    chunks = _as_chunks(k_chunks)
    _check_keys(chunks)
    k = _kv_like(chunks)
    B, N, Hkv, D = k.shape
    blocks = -(-N // block_len) if block_len > 0 else 0
    if means is None:
        means = torch.zeros((B, Hkv, blocks, D), device=chunks[0].device, dtype=torch.float32)
    _check_means(means, B, Hkv, blocks, D)
    _check_device(means, *chunks)
    one = torch.Size((B, 1, Hkv, D))
    p = AttnParams(B, 1, Hkv, Hkv, D, 1, N, 0, kv_begin, kv_end, 1.0, BF16, *_contiguous_strides(one), *k.stride()[:3], *_contiguous_strides(one),
                   *_contiguous_strides(one))
    _check(lib.slimpipe_attn_block_means(ctypes.byref(p), _chunk_table(chunks), len(chunks), chunks[0].shape[1], block_len, means.data_ptr(),
                                         _stream()), "slimpipe_attn_block_means")
    return means


def _contiguous_strides(shape):
    return shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3]


def slimpipe_attn_block_select(q_slice, means, q_offset, kv_begin, kv_end, block_len, top_k, causal=True, index=None):
    """-> index [B, Hq, s, top_k] int32: the blocks of every query row, ascending, filled up with -1."""
    shape = q_slice.shape
    _check_rows("q_slice", q_slice, shape)
    if means.dim() != 4:
        raise SlimpipeError("means must have four dimensions")
    B, s, Hq, D = shape
    Hkv, blocks = means.shape[1], means.shape[2]
    _check_means(means, B, Hkv, blocks, D)
    if index is None:
        index = torch.empty((B, Hq, s, top_k), device=q_slice.device, dtype=torch.int32)
    if _check_index(index, shape) != top_k:
        raise SlimpipeError("index must have top_k entries a row")
    _check_device(q_slice, means, index)
    sq = q_slice.stride()
    p = AttnParams(B, s, Hq, Hkv, D, 1 if causal else 0, blocks * block_len, q_offset, kv_begin, kv_end, 1.0, BF16, sq[0], sq[1], sq[2],
                   Hkv * D, Hkv * D, D, sq[0], sq[1], sq[2], sq[0], sq[1], sq[2])
    _check(lib.slimpipe_attn_block_select(ctypes.byref(p), q_slice.data_ptr(), means.data_ptr(), block_len, top_k, index.data_ptr(), _stream()),
           "slimpipe_attn_block_select")
    return index


def _block_ws(p, block_len, top_k, is_bwd):
    n = ctypes.c_size_t(0)
    _check(lib.slimpipe_attn_block_workspace_bytes(ctypes.byref(p), block_len, top_k, 1 if is_bwd else 0, ctypes.byref(n)), "block_workspace_bytes")
    return n.value


def slimpipe_attn_block_workspace_bytes(q_slice, k_chunks, index, q_offset, kv_begin, kv_end, block_len, causal=True, is_bwd=False):
    """Bytes of workspace that slimpipe_attn_block_fwd (or _bwd) of these tensors needs."""
    k_chunks = _as_chunks(k_chunks)
    shape = q_slice.shape
    # (sizes alone: nothing is read, so stand-ins of any dtype will do)
    _check_rows("q_slice", q_slice, shape, q_slice.dtype)
    _check_keys(k_chunks, shape, k_chunks[0].dtype if k_chunks else None)
    p = _params(q_slice, _kv_like(k_chunks), q_slice, q_slice, q_offset, kv_begin, kv_end, causal, None, BF16)
    return _block_ws(p, block_len, _check_index(index, shape), is_bwd)


def slimpipe_attn_block_fwd(q_slice, k_chunks, v_chunks, index, q_offset, kv_begin, kv_end, block_len, causal=True, scale=None, out_dtype=BF16,
                            out=None, lse=None, workspace=None):
    """-> (out, lse): slimpipe_attn_fwd restricted to the keys of the blocks that `index` names for each row.  k_chunks / v_chunks: one
    tensor each or lists of chunks.  workspace: uint8 tensor, allocated where None."""
    k_chunks, v_chunks = _as_chunks(k_chunks), _as_chunks(v_chunks)
    shape = q_slice.shape
    _check_rows("q_slice", q_slice, shape)
    _check_keys(k_chunks, shape)
    _check_keys(v_chunks)
    top_k = _check_index(index, shape)
    if len(k_chunks) != len(v_chunks) or not _same_strides(v_chunks[0], k_chunks[0]):
        raise SlimpipeError("v must have as many chunks as k, of the same shape and strides")
    if out is None or lse is None:
        out, lse = _outputs(q_slice, out_dtype, out, lse)
    _check_rows("out (its dtype is out_dtype's)", out, shape, _TORCH_DTYPE.get(out_dtype))
    _check_lse(lse, shape)
    p = _params(q_slice, _kv_like(k_chunks), out, out, q_offset, kv_begin, kv_end, causal, scale, out_dtype)
    if workspace is None:
        workspace = torch.empty(_block_ws(p, block_len, top_k, False), device=q_slice.device, dtype=torch.uint8)
    _check_workspace(workspace)
    _check_device(q_slice, index, out, lse, workspace, *k_chunks, *v_chunks)
    _check(lib.slimpipe_attn_block_fwd(ctypes.byref(p), q_slice.data_ptr(), _chunk_table(k_chunks), _chunk_table(v_chunks), len(k_chunks),
                                       k_chunks[0].shape[1], block_len, top_k, index.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                       *_ws(workspace), _stream()), "slimpipe_attn_block_fwd")
    return out, lse


def slimpipe_attn_block_bwd(q_slice, k_chunks, v_chunks, index, out, d_out, lse, q_offset, kv_begin, kv_end, block_len, dk_chunks, dv_chunks,
                            causal=True, scale=None, dq=None, dq_dtype=BF16, dq_accumulate=False, dkv_accumulate=True, workspace=None):
    """-> dq: the gradients of slimpipe_attn_block_fwd with the same index.  dk_chunks / dv_chunks (fp32, one tensor each or lists, shaped like
    the keys) get rows [kv_begin, kv_end) written or incremented."""
    k_chunks, v_chunks, dk_chunks, dv_chunks = (list(_as_chunks(x)) for x in (k_chunks, v_chunks, dk_chunks, dv_chunks))
    shape = q_slice.shape
    _check_rows("q_slice", q_slice, shape)
    _check_keys(k_chunks, shape)
    top_k = _check_index(index, shape)
    if dq is None:
        # (the strides of q also where those leave gaps: a slice of a sequence, a part of packed rows)
        dq = torch.empty_strided(q_slice.shape, q_slice.stride(), device=q_slice.device, dtype=torch.float32 if dq_dtype == F32 else torch.bfloat16)
    if not _same_strides(dq, q_slice):
        raise SlimpipeError("dq must have the strides of q")
    for c in v_chunks + dk_chunks + dv_chunks:
        if not _same_strides(c, k_chunks[0]):
            raise SlimpipeError("v, dk and dv must have the strides of k")
    if not len(k_chunks) == len(v_chunks) == len(dk_chunks) == len(dv_chunks):
        raise SlimpipeError("k, v, dk and dv must have the same number of chunks")
    _check_keys(v_chunks)
    _check_keys(dk_chunks + dv_chunks, None, torch.float32)
    _check_rows("dq (its dtype is dq_dtype's)", dq, shape, _TORCH_DTYPE.get(dq_dtype))
    _check_rows("out", out, shape)
    _check_rows("d_out", d_out, shape)
    _check_lse(lse, shape)
    p = _params(q_slice, _kv_like(k_chunks), out, d_out, q_offset, kv_begin, kv_end, causal, scale, BF16)
    if workspace is None:
        workspace = torch.empty(_block_ws(p, block_len, top_k, True), device=q_slice.device, dtype=torch.uint8)
    _check_workspace(workspace)
    _check_device(q_slice, index, out, d_out, lse, dq, workspace, *k_chunks, *v_chunks, *dk_chunks, *dv_chunks)
    _check(lib.slimpipe_attn_block_bwd(ctypes.byref(p), q_slice.data_ptr(), _chunk_table(k_chunks), _chunk_table(v_chunks), len(k_chunks),
                                       k_chunks[0].shape[1], block_len, top_k, index.data_ptr(), out.data_ptr(), d_out.data_ptr(), lse.data_ptr(),
                                       dq.data_ptr(), dq_dtype, 1 if dq_accumulate else 0, _chunk_table(dk_chunks), _chunk_table(dv_chunks),
                                       1 if dkv_accumulate else 0, *_ws(workspace), _stream()), "slimpipe_attn_block_bwd")
    return dq


class KvCache4(collections.namedtuple("KvCache4", "k_codes k_scales v_codes v_scales")):
    """A key/value cache held in 4 bits: uint8 tensors [B, capacity, Hkv, D / 2] (codes) and [B, capacity, Hkv, D / 32] (scales)."""
    __slots__ = ()

    @classmethod
    def empty(cls, batch, capacity, kv_heads, head_dim, device="cuda"):
        def new(n):
            return torch.zeros((batch, capacity, kv_heads, n), device=device, dtype=torch.uint8)
        return cls(new(head_dim // 2), new(head_dim // 32), new(head_dim // 2), new(head_dim // 32))

    def layout(self):
        """(batch, capacity, kv heads, head_dim) and the three strides in elements, after a check that the four tensors agree."""
        kc, ks, vc, vs = self
        shape, codes, scales, v_codes, v_scales = kc.shape, kc.stride(), ks.stride(), vc.stride(), vs.stride()
        u8 = torch.uint8
        if codes[3:] == scales[3:] == v_codes[3:] == v_scales[3:] == (1,) and kc.dtype is ks.dtype is vc.dtype is vs.dtype is u8 and vc.shape == shape:
            B, N, H, half = shape
            b, n, h = codes[:3]
            # (a dimension of one element may have any stride)
            if (ks.shape == vs.shape == (B, N, H, half // 16) and (B == 1 or b == v_codes[0] == 16 * scales[0] == 16 * v_scales[0])
                    and (N == 1 or n == v_codes[1] == 16 * scales[1] == 16 * v_scales[1]) and (H == 1 or h == v_codes[2] == 16 * scales[2] == 16 * v_scales[2])):
                D = 2 * half
                return (B, N, H, D), (2 * b if B > 1 else N * H * D, 2 * n if N > 1 else H * D, 2 * h if H > 1 else D)
        raise SlimpipeError("codes and scales must be uint8 [batch, keys, heads, head_dim / 2] and [.., head_dim / 32] of the same layout")


def _cache_ptrs(cache):
    return cache.k_codes.data_ptr(), cache.k_scales.data_ptr(), cache.v_codes.data_ptr(), cache.v_scales.data_ptr()


def slimpipe_attn_kv4_store(k_slice, v_slice, cache, position):
    """Store bf16 rows k_slice, v_slice [B, s, Hkv, D] in a KvCache4 from `position` on."""
    (B, N, H, D), skv = cache.layout()
    if tuple(k_slice.shape) != (B, k_slice.shape[1], H, D) or k_slice.stride(3) != 1 or not _same_strides(k_slice, v_slice):
        raise SlimpipeError("k_slice and v_slice must be [batch, rows, kv heads, head_dim] of the cache, with the same strides")
    if not k_slice.dtype is v_slice.dtype is torch.bfloat16:
        raise SlimpipeError("k_slice and v_slice must be torch.bfloat16")
    _check_device(k_slice, v_slice, *cache)
    sx = k_slice.stride()[:3]
    p = AttnParams(B, k_slice.shape[1], H, H, D, 1, N, position, 0, 0, 1.0, BF16, *sx, *skv, *sx, *sx)
    _check(lib.slimpipe_attn_kv4_store(ctypes.byref(p), k_slice.data_ptr(), v_slice.data_ptr(), *_cache_ptrs(cache), _stream()), "slimpipe_attn_kv4_store")


def slimpipe_attn_kv4_load(cache, kv_begin, kv_end, k_rows=None, v_rows=None):
    """-> (k, v) bf16 [B, kv_end - kv_begin, Hkv, D]: the numbers that the rows of a KvCache4 stand for."""
    (B, N, H, D), skv = cache.layout()
    if kv_end < kv_begin:
        raise SlimpipeError("kv_end lies before kv_begin")
    shape = (B, kv_end - kv_begin, H, D)
    if k_rows is None and v_rows is None:
        k_rows, v_rows = torch.empty((2,) + shape, device=cache.k_codes.device, dtype=torch.bfloat16).unbind(0)
    else:
        if k_rows is None:
            k_rows = torch.empty_strided(v_rows.shape, v_rows.stride(), device=v_rows.device, dtype=v_rows.dtype)      # (gaps and all)
        elif v_rows is None:
            v_rows = torch.empty_strided(k_rows.shape, k_rows.stride(), device=k_rows.device, dtype=k_rows.dtype)
        if tuple(k_rows.shape) != shape or k_rows.stride(3) != 1 or not _same_strides(k_rows, v_rows):
            raise SlimpipeError("k_rows and v_rows must be [batch, kv_end - kv_begin, kv heads, head_dim] with the same strides")
        if not k_rows.dtype is v_rows.dtype is torch.bfloat16:
            raise SlimpipeError("k_rows and v_rows must be torch.bfloat16")
    _check_device(k_rows, v_rows, *cache)
    sx = k_rows.stride()[:3] if shape[1] > 0 else (H * D, H * D, D)
    p = AttnParams(B, 1, H, H, D, 1, N, 0, kv_begin, kv_end, 1.0, BF16, *sx, *skv, *sx, *sx)
    _check(lib.slimpipe_attn_kv4_load(ctypes.byref(p), *_cache_ptrs(cache), k_rows.data_ptr() or None, v_rows.data_ptr() or None, _stream())
           if shape[1] > 0 else lib.slimpipe_attn_validate(ctypes.byref(p), 0), "slimpipe_attn_kv4_load")
    return k_rows, v_rows


def _kv4_params(q_slice, cache, out_like, q_offset, kv_begin, kv_end, causal, scale, out_dtype):
    (B, N, H, D), skv = cache.layout()
    shape = q_slice.shape
    if len(shape) != 4 or shape[0] != B or shape[3] != D:
        raise SlimpipeError("q_slice and the cache must have the same batch and head_dim")
    sq, so = q_slice.stride(), out_like.stride()
    return AttnParams(B, shape[1], shape[2], H, D, 1 if causal else 0, N, q_offset, kv_begin, kv_end,
                      float(scale) if scale is not None else 1.0 / math.sqrt(D), out_dtype, *sq[:3], *skv, *so[:3], *so[:3])


def _kv4_ws(p):
    n = ctypes.c_size_t(0)
    _check(lib.slimpipe_attn_kv4_workspace_bytes(ctypes.byref(p), ctypes.byref(n)), "kv4_workspace_bytes")
    return n.value


def slimpipe_attn_kv4_workspace_bytes(q_slice, cache, q_offset, kv_begin, kv_end, causal=True):
    """Bytes of workspace that slimpipe_attn_fwd_kv4 of these tensors needs (may be 0)."""
    return _kv4_ws(_kv4_params(q_slice, cache, q_slice, q_offset, kv_begin, kv_end, causal, None, BF16))


def slimpipe_attn_fwd_kv4(q_slice, cache, q_offset, kv_begin, kv_end, causal=True, scale=None, out_dtype=BF16, out=None, lse=None, workspace=None):
    """-> (out, lse): slimpipe_attn_fwd over a KvCache4.  workspace: uint8 tensor, allocated where None."""
    shape = q_slice.shape
    _check_rows("q_slice", q_slice, shape)
    if out is None or lse is None:
        out, lse = _outputs(q_slice, out_dtype, out, lse)
    _check_rows("out (its dtype is out_dtype's)", out, shape, _TORCH_DTYPE.get(out_dtype))
    _check_lse(lse, shape)
    p = _kv4_params(q_slice, cache, out, q_offset, kv_begin, kv_end, causal, scale, out_dtype)
    if workspace is None:
        workspace = torch.empty(_kv4_ws(p), device=q_slice.device, dtype=torch.uint8)
    _check_workspace(workspace)
    _check_device(q_slice, out, lse, workspace, *cache)
    _check(lib.slimpipe_attn_fwd_kv4(ctypes.byref(p), q_slice.data_ptr(), *_cache_ptrs(cache), out.data_ptr(), lse.data_ptr(), *_ws(workspace),
                                     _stream()), "slimpipe_attn_fwd_kv4")
    return out, lse


KERNEL_KINDS = ("fwd", "delta", "dq", "dkdv", "merge", "finalize", "dkdv_reduce", "dq_reduce",
                "bwd_both", "both_reduce")


def slimpipe_attn_mfma_rate(random_operands):
    """-> TFLOP/s of a pure bf16 MFMA stream on this GPU (constant or random operands)."""
    sink = torch.zeros(4, device="cuda", dtype=torch.float32)
    tf = ctypes.c_double(0.0)
    _check(lib.slimpipe_attn_mfma_rate(1 if random_operands else 0, sink.data_ptr(), ctypes.byref(tf), _stream()), "mfma_rate")
    return tf.value


def slimpipe_attn_dq_atomic_probe(s_q, heads, key_tiles, rows_per_step, placement, rotate, filler_mfma, with_atomics):
    """-> (ms, every element of dq holds the expected count, workgroups not on XCD w % 8 [placement 1 only])."""
    dq = torch.zeros((s_q, heads, 128), device="cuda", dtype=torch.float32)
    mism = torch.zeros(1, device="cuda", dtype=torch.int32)
    ms = ctypes.c_double(0.0)
    torch.cuda.synchronize()
    rc = lib.slimpipe_attn_dq_atomic_probe(dq.data_ptr(), s_q, heads, key_tiles, rows_per_step, placement, rotate, filler_mfma,
                                           1 if with_atomics else 0, mism.data_ptr(), ctypes.byref(ms), _stream())
    _check(rc, "dq_atomic_probe (step/HIP error %s)" % ms.value)
    want = float(key_tiles * (64 // rows_per_step)) if with_atomics else 0.0
    ok = bool((dq == want).all())
    return ms.value, ok, int(mism.item())


def slimpipe_attn_xcd_rate(iters=20000, rounds=4):
    """-> {xcd: (workgroups, mean workgroup ms, last end ms)} for `rounds` workgroups of equal matrix work per compute unit."""
    n = rounds * torch.cuda.get_device_properties(0).multi_processor_count
    t0 = torch.zeros(n, device="cuda", dtype=torch.int64)
    t1 = torch.zeros(n, device="cuda", dtype=torch.int64)
    xcc = torch.zeros(n, device="cuda", dtype=torch.int32)
    for _ in range(2):          # the second launch is the one reported (clocks settled)
        _check(lib.slimpipe_attn_xcd_rate(iters, n, t0.data_ptr(), t1.data_ptr(), xcc.data_ptr(), _stream()), "xcd_rate")
    t0, t1, xcc = t0.cpu(), t1.cpu(), xcc.cpu()
    base = int(t0.min())
    out = {}
    for x in sorted(set(xcc.tolist())):
        sel = xcc == x
        out[int(x)] = (int(sel.sum()), float((t1[sel] - t0[sel]).double().mean()) / 1e5, float(int(t1[sel].max()) - base) / 1e5)
    return out


def slimpipe_attn_bwd_plan(params, n_chunks, workspace_bytes):
    """How a backward call would be cut into work items with a workspace of that size (host code only)."""
    plan = BwdPlan()
    _check(lib.slimpipe_attn_bwd_plan(ctypes.byref(params), n_chunks, workspace_bytes, ctypes.byref(plan)), "bwd_plan")
    return plan


def slimpipe_attn_call_path(params, is_bwd, n_chunks, workspace_bytes):
    """Which kernels a call with a workspace of that size takes (host code only; forward: 0 bytes = no workspace)."""
    path = CallPath()
    _check(lib.slimpipe_attn_call_path(ctypes.byref(params), 1 if is_bwd else 0, n_chunks, workspace_bytes, ctypes.byref(path)), "call_path")
    return path


def slimpipe_attn_small_bwd_plan(params, n_chunks, workspace_bytes):
    """How the kernel of 32-row and 32-key items would do a backward call that takes it; all zero for others (host code only)."""
    plan = SmallBwdPlan()
    _check(lib.slimpipe_attn_small_bwd_plan(ctypes.byref(params), n_chunks, workspace_bytes, ctypes.byref(plan)), "small_bwd_plan")
    return plan


def slimpipe_attn_profile_enable(enable):
    _check(lib.slimpipe_attn_profile_enable(1 if enable else 0), "profile_enable")


def slimpipe_attn_profile_read():
    """-> {kernel kind: (total ms, launches)} since the last read (waits for the recorded events)."""
    ms = (ctypes.c_double * len(KERNEL_KINDS))()
    n = (ctypes.c_int64 * len(KERNEL_KINDS))()
    _check(lib.slimpipe_attn_profile_read(ms, n), "profile_read")
    return {k: (ms[i], n[i]) for i, k in enumerate(KERNEL_KINDS)}
