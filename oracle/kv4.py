"""A K/V cache in 4 bits (oracle; test infrastructure).

Rows of 128 values in blocks of 32 that share a power of two 2^e, elements in
E2M1: sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6. A block with largest
magnitude `top` takes the smallest e with top <= 7 * 2^e in [-124, 125] (-124
for zeros), each element the nearest value of x / 2^e, ties to the even code,
magnitudes over 6 to 6. A block with a NaN or an infinity becomes NaN.

Everything is float64 and written from that definition by search: the exponent
is found by trial, an element by comparing distances.
"""

from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
E_MIN, E_MAX, NAN_BYTE = -124, 125, 255


def block_exponent(top: float) -> int:
    e = E_MIN
    while e < E_MAX and top > 7.0 * 2.0 ** e:
        e += 1
    return e


def nearest_code(x: float) -> int:
    """Code of the E2M1 value nearest to x, ties to the even code, saturating."""
    off = np.abs(LEVELS - abs(x))
    best = np.flatnonzero(off == off.min())
    code = int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])
    return code | (8 if np.signbit(x) else 0)


def quantise(rows):
    """rows [..., D] -> codes uint8 [..., D/2] (even element in the low half),
    scale bytes uint8 [..., D/32]. Codes of NaN blocks are 0."""
    rows = np.asarray(rows, np.float64)
    D = rows.shape[-1]
    flat = rows.reshape(-1, BLOCK)
    codes = np.zeros(flat.shape, np.uint8)
    scales = np.zeros(len(flat), np.uint8)
    for i, x in enumerate(flat):
        if not np.isfinite(x).all():
            scales[i] = NAN_BYTE
            continue
        e = block_exponent(np.abs(x).max())
        scales[i] = e + 127
        codes[i] = [nearest_code(v) for v in x / 2.0 ** e]
    codes = codes.reshape(*rows.shape[:-1], D // 2, 2)
    return codes[..., 0] | codes[..., 1] << 4, scales.reshape(*rows.shape[:-1], D // BLOCK)


def values(codes, scales):
    """The float64 values that codes [..., D/2] and scale bytes [..., D/32] stand for."""
    codes, scales = np.asarray(codes, np.uint8), np.asarray(scales, np.uint8)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, BLOCK)
    x = LEVELS[c & 7] * np.where(c & 8, -1.0, 1.0)
    f = np.where(scales == NAN_BYTE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (x * f[..., None]).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def write_tokens(cache, rows, table, position: int):
    """Quantise one tensor's rows [n, heads, D] to positions position .. + n - 1
    of a request; cache = (codes [pages, heads, 16, D/2], scales), in place."""
    codes, scales = quantise(rows)
    for t in range(len(rows)):
        page, at = int(table[(position + t) // 16]), (position + t) % 16
        cache[0][page, :, at], cache[1][page, :, at] = codes[t], scales[t]
