"""An 8-bit paged cache on the host, from its definition: e4m3 codes by nearest
value over the type's own table, scales as whole exponents.

Everything here is exact (values of a few bits times powers of two), and so is what
the kernels do: codes and scales are compared for equality."""
from __future__ import annotations

import numpy as np
import torch

LEAST = -117  # exponents of scales


def _grid():
    e, m = np.divmod(np.arange(127), 8)
    return np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)


GRID = _grid()
MID = (GRID[1:] + GRID[:-1]) / 2


def decode(codes):
    """uint8 codes -> values (NaN for 0x7f and 0xff)."""
    v = np.append(GRID, np.nan)[codes & 127]
    return np.where(codes & 128, -v, v)


def encode(x):
    """The nearest codes of |x| <= 448, ties to the even one; 0x7f where x is not finite."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.size == 0 or a.max() <= 448
    low, high = np.searchsorted(MID, a, "left"), np.searchsorted(MID, a, "right")
    c = np.where(low % 2 == 0, low, high)
    return np.where(np.isfinite(x), c | np.where(np.signbit(x), 128, 0), 127).astype(np.uint8)


def exponent(x):
    """The least e with max |x| <= 448 2^e over the finite entries, >= LEAST."""
    m = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = LEAST
    if m > 0:
        f, p = np.frexp(m / 448)
        e = max(e, int(p) - (f == 0.5))
    return e


def write(pool, scales, x, table, first, start):
    """One pool's codes [n][page][H][d] and scales' bytes [n][blocks][H], changed in place, for
    rows x [N][H][d]."""
    n_pages, page, H, _ = pool.shape
    sb, cap, N = page // scales.shape[1], table.shape[1] * page, len(x)
    at = np.clip(start, 0, N)
    at[0] = 0
    for b in range(len(first)):
        p0 = int(np.clip(first[b], 0, cap))
        p1 = min(p0 + max(int(at[b + 1] - at[b]), 0), cap)
        p = p0
        while p < p1:
            end = min(p // sb * sb + sb, p1)
            pg, i = int(table[b, p // page]), p % page
            if 0 <= pg < n_pages:
                rows = x[at[b] + p - p0:at[b] + end - p0]
                for h in range(H):
                    e = exponent(rows[:, h])
                    s = (pg, i // sb, h)
                    if p % sb:
                        old = int(scales[s]) - 127
                        e = max(e, old)
                        live = slice(i - p % sb, i)
                        if e > old:
                            v = decode(pool[pg, live, h])
                            c = encode(v * 2.0 ** (old - e))
                            pool[pg, live, h] = np.where(np.isnan(v), pool[pg, live, h] & 128 | 127, c)
                    scales[s] = e + 127
                    pool[pg, i:i + end - p, h] = encode(rows[:, h] * 2.0 ** -float(e))
            p = end


def values(pool, scales):
    """Codes and scales' bytes -> values."""
    sb = pool.shape[1] // scales.shape[1]
    return decode(pool) * (2.0 ** (scales.astype(np.float64) - 127)).repeat(sb, 1)[..., None]


class Cache:
    """An 8-bit cache on the device; k and v start as codes and scales of anything."""

    def __init__(self, n_pages, page, sb, Hkv, d, seed=0):
        r = np.random.RandomState(seed)
        self.host = {}
        for x in "kv":
            codes = r.randint(0, 256, (n_pages, page, Hkv, d)).astype(np.uint8)
            self.host[x] = codes, r.randint(100, 140, (n_pages, page // sb, Hkv)).astype(np.uint8)
        self.send()

    def send(self):
        self.k, self.v = (torch.from_numpy(self.host[x][0]).cuda().view(torch.float8_e4m3fn) for x in "kv")
        self.ks, self.vs = (torch.from_numpy(self.host[x][1]).cuda().view(torch.float8_e8m0fnu) for x in "kv")

    @property
    def args(self):
        return self.k, self.v, self.ks, self.vs

    def codes(self, x):
        """(codes, scales' bytes) of the device's k or v."""
        p, s = (self.k, self.ks) if x == "k" else (self.v, self.vs)
        return p.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()
