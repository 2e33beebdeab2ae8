"""Microscaled messages in 64 bits with numpy, from their definition: the reference of the tests of
the adpsgd_mx_* calls."""
import numpy as np

E2M1, E4M3 = 0, 1


def grid(fmt):
    """The non-negative numbers of a format by code (E4M3's code 127 is NaN)."""
    if fmt == E2M1:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    g = [m * 2.0 ** -9 for m in range(8)]
    g += [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
    return np.array(g[:-1] + [np.nan])


def difference(x, base=None, residual=None):
    """fl32(fl32(x - base) + residual), float32 [K, P]."""
    with np.errstate(all="ignore"):
        d = x if base is None else x - base
        d = d if residual is None else d + residual
    return d.astype(np.float32)


def quantize(d, fmt):
    """codes [K, blocks, 32] (numbers 0..15 or 0..255), scale bytes [K, blocks] and the sent values
    [K, P] in 64 bits of float32 rows d."""
    K, P = d.shape
    n = -(-P // 32)
    b = np.zeros((K, n * 32))
    b[:, :P] = d
    b = b.reshape(K, n, 32)
    g = grid(fmt)[:8] if fmt == E2M1 else grid(fmt)[:127]
    most = np.abs(b).max(-1)                       # (NaN if the block holds one)
    bad = ~np.isfinite(most)
    e = np.full(most.shape, -127)
    for cand in range(-126, 128):                  # the least power of two that holds the largest
        e = np.where(np.where(bad, 0, most) > g[-1] * 2.0 ** (cand - 1), cand, e)
    byte = np.where(bad, 255, e + 127)
    s = np.ldexp(1.0, e)[..., None]
    v = np.where(bad[..., None], 0.0, b)
    a = np.abs(v) / s
    i = np.clip(np.searchsorted(g, a), 1, len(g) - 1)
    lo, hi = g[i - 1], g[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))     # ties to the even code
    c = np.where(up, i, i - 1)
    c = np.where(g[c] * s >= 2.0 ** 128, c - 1, c)                   # (no fp32 number)
    val = np.where(np.signbit(v), -1.0, 1.0) * g[c] * s
    val[bad] = np.nan
    codes = c + np.where(np.signbit(v), 8 if fmt == E2M1 else 128, 0)
    return codes, byte, val.reshape(K, -1)[:, :P]


def pack(codes, fmt):
    """uint8 [K, bytes] of code numbers [K, blocks, 32]."""
    c = codes.reshape(codes.shape[0], -1).astype(np.uint8)
    return c if fmt == E4M3 else (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)


def values(codes, byte, P, fmt):
    """What codes [K, bytes] with scale bytes [K, blocks] say, in 64 bits [K, P]."""
    K, n = codes.shape[0], -(-P // 32)
    c = codes.astype(np.int64)
    if fmt == E2M1:
        c = np.stack([c & 15, c >> 4], -1).reshape(K, -1)
    half = 8 if fmt == E2M1 else 128
    v = grid(fmt)[c % half] * np.where(c >= half, -1.0, 1.0)
    s = np.ldexp(1.0, byte[:, :n].astype(np.int64) - 127)
    s[byte[:, :n] == 255] = np.nan
    return (v[:, :n * 32].reshape(K, n, 32) * s[..., None]).reshape(K, -1)[:, :P]


def average(v, off, base=None):
    """(base + mean [P], variance of every tensor [T]) of rows v in 64 bits."""
    mean = v.mean(0)
    new = mean if base is None else base.astype(np.float64) + mean
    dev = ((v - mean) ** 2).sum(0) / v.shape[0]
    return new, np.array([dev[a:b].sum() for a, b in zip(off[:-1], off[1:])])


def product(v, w, off):
    """([T, K, K] inner products, the same of magnitudes)."""
    spans = list(zip(off[:-1], off[1:]))
    return (np.array([v[:, a:b] @ w[:, a:b].T for a, b in spans]),
            np.array([np.abs(v[:, a:b]) @ np.abs(w[:, a:b]).T for a, b in spans]))
