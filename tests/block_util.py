"""Plain 64-bit definitions of sparse attention over selected key blocks, with the error that rounding may cause.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value.  Probabilities (and dS in the backward) are rounded to bf16 for the
matrix unit once, sums are float32.  So an output sum_j p_j v_j is off by at most 2^-8 sum_j p_j |v_j|, and by 2^-8 of itself once more
where it is bf16.  The float32 part: a product of D terms is off by at most D 2^-24 sum |x y| and moves a probability by as much,
relatively; the bounds below carry it as `f32`, with the 2^-20 of a base-2 exponential and of a few float32 operations beside it.
"""
import numpy as np

HALF_BF16 = 2.0 ** -8


def means(k, begin, end, block):
    """k [B, N, H, D] -> {block: [B, H, D]} for the blocks with a key of [begin, end)."""
    return {j: k[:, j * block:min(end, (j + 1) * block)].mean(1) for j in range(begin // block, -(-end // block))}


def select(q, means_, offset, begin, end, block, top_k, causal):
    """q [B, s, Hq, D], means [B, Hkv, blocks, D] as the call got them -> index [B, Hq, s, top_k]."""
    B, s, Hq, D = q.shape
    group = Hq // means_.shape[1]
    index = np.full((B, Hq, s, top_k), -1, dtype=np.int64)
    in_range = range(begin // block, -(-end // block)) if end > begin else range(0)
    for b in range(B):
        for h in range(Hq):
            score = q[b, :, h] @ means_[b, h // group].T
            for r in range(s):
                own = (offset + r) // block
                free = [j for j in in_range if not causal or j < own]
                free.sort(key=lambda j: (-score[r, j], j))
                keep = [own] if causal and own in in_range else []
                keep = sorted(free[:top_k - len(keep)] + keep)
                index[b, h, r, :len(keep)] = keep
    return index


def visible(index, offset, begin, end, block, causal, N):
    """[B, Hq, s, N] truth: which keys a row sees."""
    B, Hq, s, _ = index.shape
    key = np.arange(N)
    see = (index[..., None] == key // block).any(-2) & (key >= begin) & (key < end)
    if causal:
        see &= key <= (offset + np.arange(s))[:, None]
    return see


class Reference:
    """Forward (and, given d_out, backward) in 64 bits; *_tol: how far a right result may be off, element by element."""

    def __init__(self, q, k, v, see, scale, out_bf16=True, parts_16=False):
        self.q, self.k, self.v, self.see, self.scale = q, k, v, see, scale
        B, s, Hq, D = q.shape
        g = Hq // k.shape[2]
        K, V = np.repeat(k, g, 2).transpose(0, 2, 1, 3), np.repeat(v, g, 2).transpose(0, 2, 1, 3)      # [B, Hq, N, D]
        Q = q.transpose(0, 2, 1, 3)
        K, V = np.where(see.any(2)[..., None], K, 0.0), np.where(see.any(2)[..., None], V, 0.0)         # (unseen keys may hold anything)
        self.K, self.V, self.Q, self.g = K, V, Q, g
        x = np.where(see, scale * (Q @ K.swapaxes(-1, -2)), -np.inf)
        top = x.max(-1, keepdims=True, initial=-np.inf)
        with np.errstate(divide="ignore"):
            self.lse = np.where(np.isinf(top), -np.inf, top + np.log(np.exp(x - np.where(np.isinf(top), 0.0, top)).sum(-1, keepdims=True)))
        self.p = np.where(see, np.exp(x - np.where(np.isinf(self.lse), 0.0, self.lse)), 0.0)
        # error of a scaled score in nats, the largest of the row
        e = D * 2.0 ** -24 * scale * np.where(see, np.abs(Q) @ np.abs(K).swapaxes(-1, -2), 0.0)
        self.f32 = e.max(-1, keepdims=True, initial=0.0) + 2.0 ** -20 * (4.0 + np.abs(np.where(np.isinf(self.lse), 0.0, self.lse)))
        out = self.p @ V
        mag = self.p @ np.abs(V)
        tol = mag * (HALF_BF16 + 2.0 * self.f32) + (np.abs(out) * HALF_BF16 if out_bf16 else 0.0)
        # A row folded from 16-bit results of its blocks: part b of weight w_b (their sum is 1) is float16 times a scale that brings its row's
        # largest element to 2^14, so off by 2^-11 |o_b|, or by 2^-25 2^-14 of the largest where float16 is subnormal, and
        # sum_b w_b |o_b| <= sum_j p_j |v_j|.
        self.parts_16 = parts_16
        tol = tol + (mag * 2.0 ** -11 + mag.max(-1, keepdims=True) * 2.0 ** -38 if parts_16 else 0.0)
        self.lse_tol = 2.0 * self.f32[..., 0]
        self.lse = self.lse[..., 0]
        self.out, self.out_tol = out.transpose(0, 2, 1, 3), tol.transpose(0, 2, 1, 3) * 1.01 + 1e-30

    def backward(self, out, d_out, lse, dq_bf16):
        """Gradients from the saved out and lse that the call got."""
        O, G = out.transpose(0, 2, 1, 3), d_out.transpose(0, 2, 1, 3)
        B, Hq, s, D = G.shape
        x = self.scale * (self.Q @ self.K.swapaxes(-1, -2))
        L = np.where(np.isinf(lse), 0.0, lse)[..., None]
        p = np.where(self.see & ~np.isinf(lse)[..., None], np.exp(np.where(self.see, x - L, 0.0)), 0.0)
        dp = G @ self.V.swapaxes(-1, -2) - (G * O).sum(-1, keepdims=True)
        # error of dP - delta: two float32 sums of D products
        e_dp = (D + 2) * 2.0 ** -24 * (np.abs(G) @ np.abs(self.V).swapaxes(-1, -2) + (np.abs(G) * np.abs(O)).sum(-1, keepdims=True))
        ds = p * dp
        ds_tol = np.abs(ds) * (HALF_BF16 + 2.0 * self.f32) + p * e_dp * (1.0 + HALF_BF16)
        p_tol = p * (HALF_BF16 + 2.0 * self.f32)

        def fold(x):                       # query heads of a group onto their kv head, [B, N, Hkv, D]
            return x.reshape(B, Hq // self.g, self.g, x.shape[2], D).sum(2).transpose(0, 2, 1, 3)
        t = np.swapaxes
        dq = (self.scale * ds @ self.K).transpose(0, 2, 1, 3)
        dq_tol = (self.scale * ds_tol @ np.abs(self.K)).transpose(0, 2, 1, 3) * 1.01 + (np.abs(dq) * HALF_BF16 if dq_bf16 else 0.0)
        if self.parts_16 and dq_bf16:      # added up from 16-bit parts of its blocks: sum_b |dq_b| <= scale sum_j |dS_j| |k_j|
            dq_mag = (self.scale * np.abs(ds) @ np.abs(self.K)).transpose(0, 2, 1, 3) * 1.01
            dq_tol = dq_tol + 2.0 ** -11 * dq_mag + 2.0 ** -38 * dq_mag.max(-1, keepdims=True)
        # (float32 sums over rows: n 2^-24 of the summed magnitudes, below 2^-12 of what one bf16 rounding of each term may give)
        dk, dv = fold(self.scale * t(ds, -1, -2) @ self.Q), fold(t(p, -1, -2) @ G)
        dk_tol, dv_tol = fold(self.scale * t(ds_tol, -1, -2) @ np.abs(self.Q)) * 1.01, fold(t(p_tol, -1, -2) @ np.abs(G)) * 1.01
        return (dq, dq_tol + 1e-30), (dk, dk_tol + 1e-30), (dv, dv_tol + 1e-30)


def check(name, got, want, tol):
    """Equal where `want` is infinite, within `tol` elsewhere; no NaN."""
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), name + ": rows without a key differ"
    assert np.isfinite(got[fine]).all(), name + ": not finite"
    off = np.abs(got - np.where(fine, want, 0.0))[fine] / np.broadcast_to(tol, want.shape)[fine]
    worst = float(off.max()) if off.size else 0.0
    assert worst <= 1.0, "%s: %.3g times the tolerance" % (name, worst)
    return worst
