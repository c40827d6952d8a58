"""Plain 64-bit definition of the cache in 8 bits (no attention, no GPU code)."""
import numpy as np

LEAST = -110


def levels():
    """Magnitude of codes 0 .. 126."""
    c = np.arange(127)
    e, m = c // 8, c % 8
    return np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))


def round_to(x, unit):
    """The nearest of the format's numbers under scales `unit` (broadcast), of two equally near the even code; NaN for what is not finite."""
    table = levels()
    with np.errstate(invalid="ignore"):
        y = np.abs(x) / unit
        hi = np.clip(np.searchsorted(table, y), 1, 126)
        low, high = table[hi - 1], table[hi]
        up = (y - low > high - y) | ((y - low == high - y) & (hi % 2 == 0))
        got = np.sign(x) * np.where(up, high, low) * unit
    return np.where(np.isfinite(x), got, np.nan)


def unit_of(most):
    """2^e of the smallest allowed e with most <= 448 * 2^e."""
    e = np.full(np.shape(most), LEAST)
    for i in range(LEAST, 121):
        e[np.asarray(most) > 448.0 * 2.0 ** i] = i + 1
    return 2.0 ** e


class Cache:
    """values [B, rows, H, D] and scales [B, blocks, H] of rows appended slice by slice."""

    def __init__(self, B, H, D, L):
        self.L, self.values, self.units = L, np.zeros((B, 0, H, D)), np.zeros((B, 0, H))

    def append(self, x):
        L, n, s = self.L, self.values.shape[1], x.shape[1]
        B, H = x.shape[0], x.shape[2]
        blocks = -(-(n + s) // L)
        units = np.full((B, blocks, H), 2.0 ** LEAST)
        units[:, :self.units.shape[1]] = self.units
        new = np.zeros((B, s, H, x.shape[3]))
        for j in range(n // L, blocks):
            lo, hi = max(j * L, n), min((j + 1) * L, n + s)
            part = x[:, lo - n:hi - n]
            units[:, j] = np.maximum(units[:, j], unit_of(np.where(np.isfinite(part), np.abs(part), 0.0).max((1, 3))))
            new[:, lo - n:hi - n] = round_to(part, units[:, j][:, None, :, None])
            if lo > j * L:
                self.values[:, j * L:lo] = round_to(self.values[:, j * L:lo], units[:, j][:, None, :, None])
        self.values, self.units = np.concatenate([self.values, new], 1), units
        return self

    def scales(self):
        return (np.log2(self.units) + 127).astype(np.uint8)
