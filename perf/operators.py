"""Performance cases of the operators that make attention over a long prefix read less of it: sparse attention over the
key blocks that a cheap score selects for each query, and attention over a key/value cache held in 4 bits.

A case is one of five kinds of pass:
  select    what a step does before its sparse attention: the means of the key blocks that the slice has touched, and
            for every query row and head the indices of the top_k blocks that it will read
  forward   sparse attention of one query slice over the blocks of its rows (one token or a slice)
  backward  its gradients, dk and dv rounded to bf16 at the end, as a training step takes them
  store     new keys and values of a slice written to a cache of 4 bits and the same rows read back
  cached    attention of one query slice over a cache held in 4 bits (one token or a slice)

Sparse attention.  Keys come in blocks of `block` consecutive positions.  The mean of a block is the average of the keys
that it holds so far.  A query row at position t (q_offset + row) always reads its own block t // block; of the blocks before it it
reads the top_k - 1 with the largest products of the query with the mean, equal products the lower index first.  The
indices of a row ascend and are filled up with -1.  Attention is over the keys of these blocks that the row may see.

The 4-bit format.  32 consecutive elements of a head share a scale 2^e, stored as e + 127 in 8 bits, e the smallest
integer (at least -125) with max |x| < 7 * 2^e (an all-zero group counts as the smallest e); elements are x / 2^e rounded to the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code) with a sign bit above the three bits of that code, two to a byte, the
first in the low half.

Inputs are N(0,1) rounded to bf16 (queries, keys and values behind a normalisation; upstream gradients of the same
scale).  Blocks are read unevenly, as trained models do it: the first block and recent ones often, some blocks by many
rows.  Buffers that a program allocates once and keeps (outputs, workspaces) are part of the state.
"""
import math

import torch

own = False
DEV = "cuda:0"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, rows, offset, heads, kv_heads, dim, batch=1, block=0, top_k=0, begin=0, causal=True):
    """rows: query rows of the slice; offset: global position of its first row (the keys are [begin, offset + rows))."""
    c = dict(kind=kind, rows=rows, offset=offset, heads=heads, kv_heads=kv_heads, dim=dim, batch=batch, block=block,
             top_k=top_k, begin=begin, causal=causal)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One new token of each of 4 sequences of about 128K tokens: latency.
        _case("select_token", "select", 1, 130700, 8, 1, 128, batch=4, block=256, top_k=16),
        # The last slice of 8 x 16384, 8 query heads on one key/value head (the share of one of 8 tensor-parallel GPUs).
        _case("select_slice", "select", 16384, 114688, 8, 1, 128, block=512, top_k=8),
        # The attention that goes with these two: tokens, a ragged batch of short slices with grouped heads of 64 and
        # small blocks, and a slice of a long sequence.
        _case("sparse_token_forward", "forward", 1, 130700, 8, 1, 128, batch=4, block=256, top_k=16),
        _case("sparse_ragged_forward", "forward", 1337, 2901, 12, 4, 64, batch=3, block=64, top_k=12),
        _case("sparse_slice_forward", "forward", 8192, 57344, 8, 1, 128, block=512, top_k=8),
        # Training: the same ragged batch and the same slice, backward.
        _case("sparse_ragged_backward", "backward", 1337, 2901, 12, 4, 64, batch=3, block=64, top_k=12),
        _case("sparse_slice_backward", "backward", 8192, 57344, 8, 1, 128, block=512, top_k=8),
        # The cache in 4 bits: a token of each of 16 sequences, and a slice of 4096 tokens of 40 heads.
        _case("kv4_token_store", "store", 1, 4000, 8, 8, 128, batch=16),
        _case("kv4_slice_store", "store", 4096, 16384, 40, 40, 128),
        # Attention over it: tokens of 4 sequences of 32K with 40 heads, a token behind 1M keys, and a slice of a prompt.
        _case("kv4_token_forward", "cached", 1, 32767, 40, 40, 128, batch=4),
        _case("kv4_long_token_forward", "cached", 1, 64 * 16384 - 1, 8, 1, 128),
        _case("kv4_slice_forward", "cached", 4096, 7 * 4096, 8, 1, 128),
    ]


MOST_PAIRS = 8 * 8192 * 65536                     # (query row, key) pairs that the plain forms compute, all heads
MOST_KEY_ELEMS = 4 * 32768 * 40 * 128             # elements of k or v


def draw(rng):
    while True:
        kind = rng.choice(["select", "forward", "forward", "backward", "backward", "store", "cached", "cached"])
        heads, kv_heads = rng.choice([(8, 1), (8, 1), (4, 4), (8, 2), (12, 4), (16, 16), (40, 40), (4, 1), (3, 1), (16, 1)])
        dim = rng.choice([128, 128, 128, 64])
        batch = rng.choice([1, 1, 1, 2, 3, 8])
        rows = rng.randint(1, 4) if kind != "backward" and rng.random() < 0.35 else int(round(2.0 ** rng.uniform(4.0, 13.0)))
        offset = int(round(2.0 ** rng.uniform(0.0, 17.0))) if rows < 16 else int(round(rows * (2.0 ** rng.uniform(0.0, 5.0) - 1.0)))
        block = top_k = 0
        if kind in ("select", "forward", "backward"):
            block = rng.choice([64, 64, 128, 128, 192, 256, 256, 512, 512, 1024])
            top_k = rng.choice([1, 2, 3, 4, 8, 8, 12, 16, 24])
        causal = kind not in ("forward", "cached") or rng.random() < 0.9
        # a piece of the keys, as a context exchange hands it out: early rows of a slice may see none of them
        begin = rng.randint(0, offset + rows // 2) if kind in ("forward", "backward", "cached") and rng.random() < 0.2 else 0
        c = _case(None, kind, rows, offset, heads, kv_heads, dim, batch, block, top_k, begin, causal)
        keys = offset + rows
        if batch * keys * kv_heads * dim <= MOST_KEY_ELEMS and (kind in ("select", "store") or batch * heads * rows * keys <= MOST_PAIRS):
            return c


def _pairs(c):
    """(Query row, key) pairs of the pass per batch index and query head, and blocks that a row reads at most, summed over rows."""
    end = c["offset"] + c["rows"]
    pos = torch.arange(c["offset"], end, dtype=torch.int64)
    last = pos + 1 if c["causal"] else torch.full_like(pos, end)                 # one past the last key that may be seen
    if not c["block"]:
        return int((last - c["begin"]).clamp(min=0).sum()), 0
    L = c["block"]
    there = ((last + L - 1) // L - c["begin"] // L).clamp(min=0) * (last > c["begin"])
    taken = there.clamp(max=c["top_k"])
    # whole blocks but for the last of a causal row, the row's own, and the first of a range
    tail = (last - torch.maximum((last - 1) // L * L, torch.tensor(c["begin"]))) * (there > 0)
    return int(((taken - 1).clamp(min=0) * L + tail).sum()), int(taken.sum())


def work(c):
    B, D, Hq, Hkv, s = c["batch"], c["dim"], c["heads"], c["kv_heads"], c["rows"]
    end = c["offset"] + s
    keys = end - c["begin"]
    q, lse = 2 * B * s * Hq * D, 4 * B * s * Hq
    if c["kind"] == "store":
        rows = B * s * Hkv
        return {"bytes": 2 * rows * (2 * D + 2 * (D // 2 + D // 32) + 2 * D), "flops": 4 * rows * D}
    pairs, taken = _pairs(c)
    if c["kind"] == "select":
        L = c["block"]
        blocks = -(-end // L)
        new = end - c["offset"] // L * L
        scored = sum((c["offset"] + i) // L for i in range(s))
        return {"bytes": B * Hkv * (new * D * 2 + blocks * D * 4) + q + 4 * B * Hq * s * c["top_k"],
                "flops": 2 * D * B * Hq * scored + B * Hkv * new * D}
    if c["kind"] == "cached":
        kv = 2 * B * keys * Hkv * (D // 2 + D // 32)
        return {"bytes": kv + 2 * q + lse, "flops": 4 * D * B * Hq * pairs}
    read = min(keys * Hkv, taken * Hq * c["block"])                              # key rows that are read at most
    index = 4 * B * Hq * s * c["top_k"]
    if c["kind"] == "forward":
        return {"bytes": 4 * B * read * D + index + 2 * q + lse, "flops": 4 * D * B * Hq * pairs}
    return {"bytes": 4 * B * read * D + index + 4 * q + lse + 2 * 2 * B * keys * Hkv * D, "flops": 10 * D * B * Hq * pairs}


class _State:
    pass


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    B, s, D, Hq, Hkv, off = c["batch"], c["rows"], c["dim"], c["heads"], c["kv_heads"], c["offset"]
    N = off + s
    st = _State()
    st.c, st.scale, st.ws = c, 1.0 / math.sqrt(D), None
    if c["kind"] == "store":
        # the slice as it comes out of the projections, outliers among its values as keys have them
        st.k = (torch.randn((B, s, Hkv, D), generator=g, device=DEV) * (1.0 + 7.0 * (torch.rand((D,), generator=g, device=DEV) < 0.05))).to(torch.bfloat16)
        st.v = _normal(g, B, s, Hkv, D)
        st.cache = _empty_cache(B, N, Hkv, D)
        return st
    st.q = _normal(g, B, s, Hq, D)
    st.k = _normal(g, B, N, Hkv, D)
    if c["kind"] == "select":
        # means of the blocks before the slice are in hand; the run makes those that the slice has touched
        nb, L = -(-N // c["block"]), c["block"]
        # keys of a block resemble each other, or there would be nothing to select by
        st.k += torch.randn((B, nb, Hkv, D), generator=g, device=DEV).mul_(0.5).to(torch.bfloat16).repeat_interleave(L, 1)[:, :N]
        st.means = _means(st.k, 0, N, L)
        return st
    st.v = _normal(g, B, N, Hkv, D)
    st.out = torch.empty((B, s, Hq, D), device=DEV, dtype=torch.bfloat16)
    st.lse = torch.empty((B, Hq, s), device=DEV, dtype=torch.float32)
    if c["kind"] == "cached":
        st.cache = _quantise(st.k) + _quantise(st.v)
        st.k = st.v = None
        return st
    st.index = _popular_blocks(c, g)
    if c["kind"] == "backward":
        st.do = _normal(g, B, s, Hq, D)
        st.out, st.lse = _sparse_forward(st)
        st.dk, st.dv = torch.empty_like(st.k, dtype=torch.float32), torch.empty_like(st.k, dtype=torch.float32)
        st.dq, st.dk_out, st.dv_out = torch.empty_like(st.q), torch.empty_like(st.k), torch.empty_like(st.k)
    return st


def _popular_blocks(c, g):
    """Block indices as a model picks them: its own block, the first one often, near ones, and some that many rows like."""
    B, s, Hq, L, off, K = c["batch"], c["rows"], c["heads"], c["block"], c["offset"], c["top_k"]
    end = off + s
    first, nb = c["begin"] // L, -(-end // L)
    pos = torch.arange(off, end, device=DEV)[None, None, :, None]
    j = torch.arange(first, nb, device=DEV)[None, None, None, :]
    own_block = pos // L
    like = torch.randn((B, Hq, s, nb - first), generator=g, device=DEV) + torch.randn((B, Hq, 1, nb - first), generator=g, device=DEV)
    like += 3.0 * (j == 0) + 2.0 * torch.exp2((j - own_block) / 4.0).clamp(max=1.0) + 1e6 * (j == own_block)
    if c["causal"]:
        like.masked_fill_(j > own_block, -math.inf)
    take = min(K, nb - first)
    best, at = like.topk(take, dim=-1)
    at = torch.where(best == -math.inf, nb, at + first).sort(dim=-1).values
    index = torch.full((B, Hq, s, K), -1, device=DEV, dtype=torch.int32)
    index[..., :take] = torch.where(at == nb, -1, at)
    return index


# ------------------------------------------------------------------------------------------- the plain forms

def _means(k, begin, end, block):
    """Averages of the keys of blocks begin // block ... of k [B, N, H, D] that lie before `end`, [B, H, blocks, D]."""
    x = k[:, begin:end].double()
    n = -(-x.shape[1] // block)
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * block - x.shape[1]))
    count = (end - begin - torch.arange(n, device=k.device) * block).clamp(max=block)
    return (x.unflatten(1, (n, block)).sum(2) / count[None, :, None, None]).permute(0, 2, 1, 3).float().contiguous()


def _select(st):
    c = st.c
    L, K, off, s = c["block"], c["top_k"], c["offset"], c["rows"]
    N, first = off + s, off // L * L
    st.means[:, :, first // L:] = _means(st.k, first, N, L)
    B, Hkv, nb, D = st.means.shape
    # products in 64 bits: blocks whose scores are next to each other are told apart
    q = st.q.double().permute(0, 2, 1, 3).reshape(B, Hkv, -1, D)
    score = (q @ st.means.double().transpose(2, 3)).reshape(B, -1, s, nb)
    own_block = (torch.arange(off, N, device=DEV) // L)[:, None]
    j = torch.arange(nb, device=DEV)
    score.masked_fill_(j > own_block, -math.inf).masked_fill_(j == own_block, math.inf)
    score, at = score.sort(dim=-1, descending=True, stable=True)
    at = torch.where(score == -math.inf, nb, at)[..., :K].sort(dim=-1).values
    index = torch.full((B, q.shape[1] * q.shape[2] // s, s, K), -1, device=DEV, dtype=torch.int32)
    index[..., :at.shape[-1]] = torch.where(at == nb, -1, at)
    return st.means, index


def _heads_first(x, kv_heads):
    """[B, s, H, D] -> [B, kv_heads, (H / kv_heads) * s, D] in 32 bits."""
    B, _, _, D = x.shape
    return x.float().permute(0, 2, 1, 3).reshape(B, kv_heads, -1, D)


def _hidden(c, index):
    """True where a row may not see a key of [begin, end): [B or 1, heads or 1, s, keys]."""
    begin, end = c["begin"], c["offset"] + c["rows"]
    key = torch.arange(begin, end, device=DEV)
    pos = torch.arange(c["offset"], end, device=DEV)
    hide = (key > pos[:, None])[None, None] if c["causal"] else torch.zeros((1, 1, c["rows"], end - begin), device=DEV, dtype=torch.bool)
    if index is None:
        return hide
    nb = -(-end // c["block"])
    chosen = torch.zeros(index.shape[:3] + (nb + 1,), device=DEV, dtype=torch.bool)
    chosen.scatter_(3, torch.where(index < 0, nb, index).long(), True)
    return hide | ~chosen[..., key // c["block"]]


def _scores(c, scale, q, k, index):
    """Scaled scores of the rows with the keys of the range, hidden ones -inf, and the rows in the products' order."""
    s = (q @ k.transpose(2, 3)).mul_(scale)
    B, Hkv = s.shape[:2]
    s.view(B, c["heads"], c["rows"], -1).masked_fill_(_hidden(c, index), -math.inf)
    return s


def _attend(c, scale, q, k, v, index):
    """q [B, s, Hq, D], k / v [B, keys of the range, Hkv, D] -> out, lse."""
    B, s, Hq, D = q.shape
    Hkv = k.shape[2]
    p = _scores(c, scale, _heads_first(q, Hkv), _heads_first(k, Hkv), index)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ _heads_first(v, Hkv)) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).reshape(B, Hq, s)
    return out.reshape(B, Hq, s, D).permute(0, 2, 1, 3).to(torch.bfloat16), lse


def _sparse_forward(st):
    c = st.c
    return _attend(c, st.scale, st.q, st.k[:, c["begin"]:], st.v[:, c["begin"]:], st.index)


def _sparse_backward(st):
    c = st.c
    Hkv, b = c["kv_heads"], c["begin"]
    B, s, Hq, D = st.q.shape
    q, do, k, v = _heads_first(st.q, Hkv), _heads_first(st.do, Hkv), _heads_first(st.k[:, b:], Hkv), _heads_first(st.v[:, b:], Hkv)
    lse = st.lse.reshape(B, Hkv, -1, 1)
    p = _scores(c, st.scale, q, k, st.index).sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_()
    dv = p.transpose(2, 3) @ do
    delta = (do * _heads_first(st.out, Hkv)).sum(-1, keepdim=True)
    ds = (do @ v.transpose(2, 3)).sub_(delta).mul_(p)
    del p
    dq = (ds @ k).mul_(st.scale)
    dk = (ds.transpose(2, 3) @ q).mul_(st.scale)
    st.dq.copy_(dq.reshape(B, Hq, s, D).permute(0, 2, 1, 3))
    for to, x in ((st.dk_out, dk), (st.dv_out, dv)):
        to[:, :b] = 0.0
        to[:, b:] = x.permute(0, 2, 1, 3)
    return st.dq, st.dk_out, st.dv_out


def _empty_cache(B, N, Hkv, D):
    def new(n):
        return torch.zeros((B, N, Hkv, n), device=DEV, dtype=torch.uint8)
    return new(D // 2), new(D // 32), new(D // 2), new(D // 32)


def _quantise(x):
    """bf16 [..., D] -> codes uint8 [..., D / 2] and scales uint8 [..., D / 32]."""
    g = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))                    # largest = m 2^e, 0.5 <= m < 1, or 0
    e = torch.where(m == 0, -125, e - 3 + (8.0 * m >= 7.0).to(e.dtype)).clamp(min=-125)
    y = torch.ldexp(g, -e[..., None])
    a = y.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    a = ((a / step).round() * step).clamp(max=6.0)
    code = torch.where(a < 2.0, 2.0 * a, torch.where(a < 4.0, a + 2.0, a / 2.0 + 4.0)).to(torch.uint8)
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The numbers that codes and scales stand for, in 32 bits."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    x = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)[code]
    return torch.ldexp(x.unflatten(-1, (-1, 32)), (scales.int() - 127)[..., None]).flatten(-2)


def _store(st):
    c = st.c
    at = slice(c["offset"], c["offset"] + c["rows"])
    for i, x in ((0, st.k), (2, st.v)):
        st.cache[i][:, at], st.cache[i + 1][:, at] = _quantise(x)
    return tuple(_values(st.cache[i][:, at], st.cache[i + 1][:, at]).to(torch.bfloat16) for i in (0, 2))


def _cached(st):
    c = st.c
    kc, ks, vc, vs = (x[:, c["begin"]:] for x in st.cache)
    return _attend(c, st.scale, st.q, _values(kc, ks), _values(vc, vs), None)


# ------------------------------------------------------------------------------------------- the framework's calls

def _workspace(st, sp, need):
    """The workspace that the program keeps for this call."""
    if st.ws is None:
        st.ws = torch.empty(need(sp), device=DEV, dtype=torch.uint8)
    return st.ws


def _own_run(st):
    import paper_2504_14519_amd as sp
    c = st.c
    kind, off, b, end, L, causal = c["kind"], c["offset"], c["begin"], c["offset"] + c["rows"], c["block"], c["causal"]
    if kind == "select":
        sp.slimpipe_attn_block_means(st.k, off // L * L, end, L, means=st.means)
        return st.means, sp.slimpipe_attn_block_select(st.q, st.means, off, 0, end, L, c["top_k"])
    if kind == "store":
        cache = sp.KvCache4(*st.cache)
        sp.slimpipe_attn_kv4_store(st.k, st.v, cache, off)
        return sp.slimpipe_attn_kv4_load(cache, off, end)
    if kind == "cached":
        cache = sp.KvCache4(*st.cache)
        ws = _workspace(st, sp, lambda sp: sp.slimpipe_attn_kv4_workspace_bytes(st.q, cache, off, b, end, causal))
        return sp.slimpipe_attn_fwd_kv4(st.q, cache, off, b, end, causal, st.scale, out=st.out, lse=st.lse, workspace=ws)
    ws = _workspace(st, sp, lambda sp: sp.slimpipe_attn_block_workspace_bytes(st.q, st.k, st.index, off, b, end, L, causal, kind == "backward"))
    if kind == "forward":
        return sp.slimpipe_attn_block_fwd(st.q, st.k, st.v, st.index, off, b, end, L, causal, st.scale, out=st.out, lse=st.lse, workspace=ws)
    if b:                                                   # keys before the range are not this call's
        st.dk[:, :b].zero_()
        st.dv[:, :b].zero_()
    sp.slimpipe_attn_block_bwd(st.q, st.k, st.v, st.index, st.out, st.do, st.lse, off, b, end, L, st.dk, st.dv, causal, st.scale,
                               dq=st.dq, dkv_accumulate=False, workspace=ws)
    sp.slimpipe_attn_finalize_bf16(st.dk, st.dk_out)
    sp.slimpipe_attn_finalize_bf16(st.dv, st.dv_out)
    return st.dq, st.dk_out, st.dv_out


def run(st):
    if own:
        return _own_run(st)
    return {"select": _select, "forward": _sparse_forward, "backward": _sparse_backward, "store": _store, "cached": _cached}[st.c["kind"]](st)


# ------------------------------------------------------------------------------------------- 64 bits, by the definition

def _exact_values(codes, scales):
    low, high = (codes % 16).long(), (codes // 16).long()
    table = torch.tensor([sign * v for sign in (1.0, -1.0) for v in LEVELS], dtype=torch.float64, device=DEV)
    x = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=DEV)
    x[..., 0::2], x[..., 1::2] = table[low], table[high]
    return x * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(32, -1)


def _exact_round(x):
    """x [..., 32 n] -> the nearest values of the format, with the smallest allowed scale of each group."""
    g = x.double().reshape(x.shape[:-1] + (-1, 32))
    most = g.abs().amax(-1)
    e = torch.full_like(most, -125.0)
    for exponent in range(-125, 127):
        e = torch.where(most >= 7.0 * 2.0 ** exponent, float(exponent + 1), e)
    y = g / torch.pow(2.0, e)[..., None]
    best, far = torch.zeros_like(y), torch.full_like(y, math.inf)
    for code, level in sorted(enumerate(LEVELS), key=lambda p: p[0] % 2):        # even codes first: a tie stays with them
        d = (y.abs() - level).abs()
        best, far = torch.where(d < far, level, best), torch.minimum(d, far)
    return (torch.sign(y) * best * torch.pow(2.0, e)[..., None]).reshape(x.shape)


def _exact_rows(c, index, b, h, r0, r1, keys):
    """True where rows r0 .. r1 - 1 of a head see a key."""
    pos = torch.arange(c["offset"] + r0, c["offset"] + r1, device=DEV)
    see = (keys[None, :] <= pos[:, None]) if c["causal"] else torch.ones((r1 - r0, len(keys)), dtype=torch.bool, device=DEV)
    if index is not None:
        block = keys // c["block"]
        hit = torch.zeros_like(see)
        for slot in range(index.shape[-1]):
            hit |= index[b, h, r0:r1, slot].long()[:, None] == block[None, :]
        see &= hit
    return see


def _exact_attention(c, q, k_of, v_of, index, do=None):
    """Row tile by row tile, one head at a time.  k_of(b, head): keys of the range in 64 bits.  With `do`: gradients too."""
    B, s, Hq, D = q.shape
    Hkv, end = c["kv_heads"], c["offset"] + c["rows"]
    scale, keys = 1.0 / math.sqrt(D), torch.arange(c["begin"], end, device=DEV)
    out = torch.zeros((B, s, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, s), -math.inf, dtype=torch.float64, device=DEV)
    dq = torch.zeros_like(out) if do is not None else None
    dk = torch.zeros((B, end, Hkv, D), dtype=torch.float64, device=DEV) if do is not None else None
    dv = torch.zeros_like(dk) if do is not None else None
    tile = max(1, min(s, (1 << 27) // max(1, len(keys))))
    for b in range(B):
        for h in range(Hq):
            hk = h * Hkv // Hq
            k, v = k_of(b, hk), v_of(b, hk)
            for r0 in range(0, s, tile):
                r1 = min(s, r0 + tile)
                see = _exact_rows(c, index, b, h, r0, r1, keys)
                x = torch.where(see, scale * (q[b, r0:r1, h].double() @ k.T), -math.inf)
                norm = torch.logsumexp(x, -1)
                p = torch.where(see, torch.exp(x - torch.where(see.any(-1), norm, 0.0)[:, None]), 0.0)
                o = p @ v
                out[b, r0:r1, h], lse[b, h, r0:r1] = o, norm
                if do is not None:
                    d = do[b, r0:r1, h].double()
                    ds = p * (d @ v.T - (d * o).sum(-1, keepdim=True)) * scale
                    dq[b, r0:r1, h] = ds @ k
                    dk[b, c["begin"]:, hk] += ds.T @ q[b, r0:r1, h].double()
                    dv[b, c["begin"]:, hk] += p.T @ d
    return (out, lse) if do is None else (dq, dk, dv)


def exact(c, seed):
    st = prepare(c, seed)
    kind = c["kind"]
    if kind == "store":
        return _exact_round(st.k), _exact_round(st.v)
    if kind == "cached":
        kc, ks, vc, vs = (x[:, c["begin"]:] for x in st.cache)
        return _exact_attention(c, st.q, lambda b, h: _exact_values(kc[b, :, h], ks[b, :, h]), lambda b, h: _exact_values(vc[b, :, h], vs[b, :, h]), None)
    if kind != "select":
        def of(x):
            return lambda b, h: x[b, c["begin"]:, h].double()
        return _exact_attention(c, st.q, of(st.k), of(st.v), st.index, st.do if kind == "backward" else None)
    B, s, Hq, D = st.q.shape
    L, K, Hkv, N = c["block"], c["top_k"], c["kv_heads"], c["offset"] + s
    nb = -(-N // L)
    means = torch.empty((B, Hkv, nb, D), dtype=torch.float64, device=DEV)
    for j in range(nb):
        means[:, :, j] = st.k[:, j * L:min(N, (j + 1) * L)].double().mean(1)
    kept = means.float().double()                           # what the means are kept in
    index = torch.full((B, Hq, s, K), -1, dtype=torch.int32, device=DEV)
    tile = max(1, min(s, (1 << 27) // (nb * nb)))
    j = torch.arange(nb, device=DEV)
    for b in range(B):
        for h in range(Hq):
            for r0 in range(0, s, tile):
                r1 = min(s, r0 + tile)
                mine = (torch.arange(c["offset"] + r0, c["offset"] + r1, device=DEV) // L)[:, None]
                x = st.q[b, r0:r1, h].double() @ kept[b, h * Hkv // Hq].T
                x = torch.where(j < mine, x, torch.where(j == mine, math.inf, -math.inf))
                # a block is taken when fewer than top_k are ahead of it
                ahead = ((x[:, None, :] > x[:, :, None]) | ((x[:, None, :] == x[:, :, None]) & (j[None, :] < j[:, None]))).sum(-1)
                take = (ahead < K) & (j <= mine)
                place = take.cumsum(-1) - 1
                rows, blocks = take.nonzero(as_tuple=True)
                index[b, h, r0 + rows, place[rows, blocks]] = blocks.to(torch.int32)
    return means, index
