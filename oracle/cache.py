"""Positions with several axes and the quantised KV cache: codes of the OCP Microscaling
formats with a power-of-two scale per 32 channels, in float64 (test infrastructure).
"""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# E4M3: 4 exponent bits with bias 7, 3 mantissa bits; the code 127 is NaN
E4M3 = np.array([m * 2.0 ** -9 if x == 0 else (1 + m / 8) * 2.0 ** (x - 7)
                 for x in range(16) for m in range(8)][:127])
GRID = {4: E2M1, 8: E4M3}
EXPONENTS = {4: (-125, 125), 8: (-117, 119)}


def rotary_axes(x, positions, freq, axis, pairing):
    """x [rows, heads, d]; positions [axes, rows]: pair j of a head turns by
    positions[axis[j]] * freq[j]."""
    x = np.array(x, dtype=np.float64)
    n = len(freq)
    for j in range(n):
        a, b = (j, n + j) if pairing == "halves" else (2 * j, 2 * j + 1)
        angle = np.asarray(positions, dtype=np.float64)[axis[j]] * freq[j]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        x[..., a], x[..., b] = (x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s)
    return x


def _round(a, grid):
    """Index of the value of the ascending grid nearest to each a >= 0, ties to the even
    index, what passes the last value to it."""
    up = np.minimum(np.searchsorted(grid, a), len(grid) - 1)
    dn = np.maximum(up - 1, 0)
    below, above = a - grid[dn], grid[up] - a
    return np.where((below < above) | ((below == above) & (dn % 2 == 0)), dn, up)


def quantise(x, bits):
    """(codes, scales) of x [..., d]: codes [..., d] (one a byte here), scales [..., d/32].
    A group that is not finite has the scale 255 (its codes are not defined)."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    grid = GRID[bits]
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    top = np.abs(g).max(-1)
    lo, hi = EXPONENTS[bits]
    # the least e with top <= last * 2^e, found by trying: one comparison a step
    e = np.full(top.shape, lo)
    with np.errstate(all="ignore"):
        guess = np.floor(np.log2(np.where(top > 0, top, 1.0) / grid[-1])).astype(int) - 1
        e = np.where(top > 0, guess, lo)
        for _ in range(3):
            e = e + ((top > grid[-1] * np.ldexp(1.0, e)) & (top > 0))
    e = np.clip(e, lo, hi)
    code = _round(np.minimum(np.abs(g) / np.ldexp(1.0, e)[..., None], grid[-1]), grid)
    half = 8 if bits == 4 else 128
    code = np.where(np.signbit(g), code + half, code)
    return (code.reshape(x.shape).astype(np.uint8),
            np.where(finite, e + 127, 255).astype(np.uint8))


def values(codes, scales, bits):
    """What codes [..., d] and scales [..., d/32] stand for."""
    half = 8 if bits == 4 else 128
    grid = np.append(GRID[bits], np.nan) if bits == 8 else GRID[bits]
    c = np.asarray(codes, dtype=np.int64)
    v = np.where(c >= half, -grid[c % half], grid[c % half])
    s = np.asarray(scales, dtype=np.int64)
    scale = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return v * np.repeat(scale, 32, -1)


def pack_codes(codes, bits):
    """As the cache holds them: in 4 bits two to a byte, the even element low."""
    return codes if bits == 8 else codes[..., 0::2] | codes[..., 1::2] << 4


def unpack_codes(data, bits):
    if bits == 8:
        return data
    out = np.empty(data.shape[:-1] + (2 * data.shape[-1],), dtype=np.uint8)
    out[..., 0::2], out[..., 1::2] = data & 15, data >> 4
    return out


def gather(codes, scales, table_row, n, bits):
    """The first n keys (or values) of a request: [n, Hkv, d] from the paged codes."""
    ps = codes.shape[2]
    pos = np.arange(n)
    page, at = np.asarray(table_row)[pos // ps], pos % ps
    return values(unpack_codes(codes[page, :, at], bits), scales[page, :, at], bits)


def attention(q, k, v, seen, scale):
    """Rows q [rows, Hq, d] over k, v [keys, Hkv, d]; row r sees keys [0, seen[r])."""
    rows, Hq, d = q.shape
    g = Hq // k.shape[1]
    out = np.empty((rows, Hq, d))
    for r in range(rows):
        for h in range(Hq):
            z = scale * (k[:seen[r], h // g] @ q[r, h])
            p = np.exp(z - z.max())
            out[r, h] = p @ v[:seen[r], h // g] / p.sum()
    return out
