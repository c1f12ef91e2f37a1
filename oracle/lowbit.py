"""The 8-bit operators in 64 bits, from their definitions: E4M3 values, scales by blocks of 128, the product, AdamW.

Oracle code (test infrastructure): plain numpy, no code shared with the library.
"""
from __future__ import annotations

import math

import numpy as np

# The values of the E4M3 codes 0 .. 127: four bits of exponent with bias 7, three of fraction; 127 is NaN, the largest value 448.
E4M3 = np.array([(f / 8 * 2.0 ** -6) if e == 0 else (1 + f / 8) * 2.0 ** (e - 7) for e in range(16) for f in range(8)])
E4M3[127] = math.nan


def decode(codes: np.ndarray) -> np.ndarray:
    """Values of E4M3 bytes."""
    v = E4M3[codes & 0x7F]
    return np.where(codes & 0x80, -v, v)


def nearest(x: np.ndarray) -> np.ndarray:
    """The E4M3 value nearest to x (|x| <= 448), ties to the even code; NaN for what is not finite."""
    x = np.asarray(x, np.float64)
    size = np.abs(np.where(np.isfinite(x), x, 0.0))
    grid = E4M3[:127]
    up = np.clip(np.searchsorted(grid, size), 1, 126)
    low, high = grid[up - 1], grid[up]
    take_high = (size - low > high - size) | ((size - low == high - size) & (up % 2 == 0))
    return np.where(np.isfinite(x), np.copysign(np.where(take_high, high, low), x), math.nan)


def scale_exponent(block: np.ndarray) -> int:
    """max(-127, ceil(log2(amax / 448))) over the finite entries, 0 for a block of zeros: exact, by trying powers."""
    finite = np.abs(block[np.isfinite(block)])
    amax = float(finite.max()) if finite.size else 0.0
    if amax == 0.0:
        return 0
    e = math.frexp(amax / 448.0)[1] - 2
    while math.ldexp(448.0, e) < amax:
        e += 1
    return max(e, -127)


def quantize(x: np.ndarray, kind: str) -> tuple[np.ndarray, np.ndarray]:
    """(values of the codes, scale exponents [row blocks][column blocks]) by 'rows' (1 x 128), 'cols' (128 x 1) or 'tiles'."""
    br, bc = {"rows": (1, 128), "cols": (128, 1), "tiles": (128, 128)}[kind]
    rows, cols = x.shape
    q = np.empty((rows, cols))
    s = np.zeros((-(-rows // br), -(-cols // bc)), np.int64)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = np.s_[i * br:(i + 1) * br, j * bc:(j + 1) * bc]
            s[i, j] = scale_exponent(x[at])
            q[at] = nearest(x[at] * 2.0 ** -float(s[i, j]))
    return q, s


def spread(s: np.ndarray, shape: tuple[int, int], kind: str) -> np.ndarray:
    """Scale exponents (or scales) of blocks, one for each element."""
    br, bc = {"rows": (1, 128), "cols": (128, 1), "tiles": (128, 128)}[kind]
    return np.repeat(np.repeat(s, br, 0)[:shape[0]], bc, 1)[:, :shape[1]]


def mix(x: np.ndarray) -> np.ndarray:
    """The hash of the stochastic rounding, on uint32: Chris Wellons' lowbias32 ("Prospecting for Hash Functions", 2018)."""
    x = np.asarray(x, np.uint64) & 0xFFFFFFFF
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x7FEB352D)) & np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0x846CA68B)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def noise(n: int, tensor: int, seed: int) -> np.ndarray:
    """32 random bits for each of the n elements of the tensor with this index."""
    return mix(np.arange(n, dtype=np.uint64) ^ mix(np.uint64(tensor + 1)) ^ mix(np.uint64(seed)))


def adamw(p, g, m, v, *, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(p', m', v') of one step, in 64 bits."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p - lr * weight_decay * p - lr * mh / (np.sqrt(vh) + eps), m, v


def flat_exponents(x: np.ndarray) -> np.ndarray:
    """Scale exponents of consecutive blocks of 128."""
    return np.array([scale_exponent(x[i:i + 128]) for i in range(0, len(x), 128)], np.int64)


def root_values(r: np.ndarray, exponents: np.ndarray, bits16: np.ndarray | None = None) -> np.ndarray:
    """Roots r >= 0 as 8-bit states hold them, in units of their block's scale: to nearest or, by 16 random bits, up or
    down; at least 2^-9 unless zero."""
    y = r * 2.0 ** -np.repeat(exponents, 128)[:len(r)].astype(np.float64)
    if bits16 is None:
        w = nearest(y)
    else:
        unit = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
        w = np.floor(y / unit + bits16 / 65536.0) * unit
    return np.where(y > 0, np.maximum(w, 2.0 ** -9), y)
