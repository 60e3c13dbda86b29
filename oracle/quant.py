"""Plain definition of a cache in few bits (test infrastructure only): rows of codes with a power of two for each 32 elements, value by value from the formats' ladders in 64 bits."""
from __future__ import annotations

import numpy as np

BLOCK, LEAST = 32, -117


def ladder(bits):
    """Magnitudes of the codes 0, 1, ... of a format: one or three bits behind the leading one, subnormal ones below."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    return np.array([m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])


def token_bytes(heads, dim, bits):
    return -(-(heads * dim * bits // 8 + heads * dim // BLOCK) // 16) * 16


def encode(x, bits):
    """(tokens, heads, dim) -> (tokens, token_bytes) uint8, padding 0."""
    x = np.asarray(x, np.float64)
    tokens, heads, dim = x.shape
    steps, top = ladder(bits), 2 if bits == 4 else 8
    y = x.reshape(tokens, heads * dim // BLOCK, BLOCK)
    amax = np.abs(y).max(-1)
    fine = np.isfinite(amax)
    e = np.where(fine & (amax > 0), np.frexp(np.where(fine, amax, 1.0))[1] - 1 - top, LEAST)
    e = np.maximum(e, LEAST)
    z = np.where(fine[..., None], np.abs(y), 0.0) / 2.0 ** e[..., None].astype(np.float64)
    # the nearest step, the even code of two that are equally near
    high = np.searchsorted(steps, z).clip(0, len(steps) - 1)
    low = (high - 1).clip(0)
    up, down = steps[high] - z, z - steps[low]
    code = np.where((up < down) | ((up == down) & (high % 2 == 0)), high, low)
    code = np.where(z >= steps[-1], len(steps) - 1, code)
    code = np.where(fine[..., None], code + (np.signbit(y) << (bits - 1)), 0).reshape(tokens, heads * dim).astype(np.uint8)
    if bits == 4:
        code = code[:, 0::2] | code[:, 1::2] << 4
    out = np.zeros((tokens, token_bytes(heads, dim, bits)), np.uint8)
    unit = np.where(fine, e + 127, 255).astype(np.uint8)
    out[:, :code.shape[1]], out[:, code.shape[1]:code.shape[1] + unit.shape[1]] = code, unit
    return out


def decode(rows, heads, dim, bits):
    """(..., token_bytes) uint8 -> (..., heads, dim) f64."""
    n = heads * dim * bits // 8
    code, unit = rows[..., :n], rows[..., n:n + heads * dim // BLOCK].astype(np.int64)
    if bits == 4:
        code = np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], heads * dim)
    half = 1 << (bits - 1)
    steps = np.append(ladder(bits), np.nan)
    value = np.where(code >= half, -1.0, 1.0) * steps[(code % half).astype(np.int64)]
    scale = np.where(unit == 255, np.nan, 2.0 ** (unit - 127).astype(np.float64))
    return (value.reshape(*value.shape[:-1], -1, BLOCK) * scale[..., None]).reshape(*value.shape[:-1], heads, dim)
