"""fp64 oracle of the 8-bit cache format and of rotary positions.  Test infrastructure only; shares nothing with the
CUDA path.

The e4m3 grid is written out from its definition (sign, four exponent bits with bias 7, three fraction bits; exponent
field 0 is subnormal; 0x7f and 0xff are NaN, there are no infinities), and encoding looks the nearest value up in it.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64


def _grid() -> np.ndarray:
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        mag = (f / 8.0) * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7)
        if e == 15 and f == 7:
            mag = math.nan
        v[c] = -mag if c & 128 else mag
    return v


VALUES = _grid()
_POSITIVE = VALUES[:127]     # 0 .. 448, ascending


def decode(codes: np.ndarray) -> np.ndarray:
    return VALUES[np.asarray(codes, dtype=np.uint8)]


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one, magnitudes above 448 to 448; NaN and infinities to 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    hi = np.searchsorted(_POSITIVE, mag)             # first grid value >= mag
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - mag, mag - _POSITIVE[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(_POSITIVE[hi] == mag, hi, code).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), code, 0x7f).astype(np.uint8)


def needed(a: float) -> float:
    """The smallest power of two >= a / 448, at least 2^-126."""
    s = 2.0 ** -126
    while 448.0 * s < a:
        s *= 2.0
    return s


def store(codes, scale, x, start: int, count: int):
    """One sequence and KV head: codes uint8 [cap, 128], scale [cap / 64], x float64 [T, 128].  Updates both in place."""
    end = min(start + count, codes.shape[0])
    for blk in range(start // BLOCK, (end + BLOCK - 1) // BLOCK):
        lo, hi = max(blk * BLOCK, start), min((blk + 1) * BLOCK, end)
        if hi <= lo:
            continue
        new = x[lo - start: hi - start]
        fin = np.abs(new[np.isfinite(new)])
        s = needed(fin.max() if fin.size else 0.0)
        if lo > blk * BLOCK:
            old = scale[blk]
            if s > old:
                rows = slice(blk * BLOCK, lo)
                codes[rows] = encode(decode(codes[rows]) * (old / s))
            else:
                s = old
        codes[lo:hi] = encode(new / s)
        scale[blk] = s
    return end


def values(codes, scale) -> np.ndarray:
    """float64 [n, 128] of the first n rows' codes, their blocks' scales applied."""
    return decode(codes) * np.repeat(np.asarray(scale, dtype=np.float64), BLOCK)[: codes.shape[0], None]


# ----------------------------------------------------------------------------------------------------- rotary positions
def rope_frequencies(rot, theta, scaling="none", factor=1.0, trained_len=8192, low=1.0, high=4.0, fast=32.0, slow=1.0):
    """Radians per position of the rot / 2 pairs, and the amplitude of sine and cosine."""
    f, amp = [], 1.0
    for i in range(rot // 2):
        w = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            w = w / factor
        elif scaling == "bands":
            turns = trained_len * w / (2 * math.pi)          # how often the pair turns over the trained length
            part = 1.0 if turns > high else 0.0 if turns < low else (turns - low) / (high - low)
            w = w * part + w / factor * (1 - part)
        elif scaling == "ramp":
            at = [rot * math.log(trained_len / (n * 2 * math.pi)) / (2 * math.log(theta)) for n in (fast, slow)]
            first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            part = min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
            w = w * (1 - part) + w / factor * part
            amp = 0.1 * math.log(factor) + 1.0
        f.append(w)
    return np.array(f), amp


def rope(x, pos, f, amp, layout):
    """x float64 [n, heads, 128], pos [n]: the first 2 len(f) channels of every head turned by pos * f."""
    y = np.array(x, dtype=np.float64)
    r = len(f)
    a = np.asarray(pos, dtype=np.float64)[:, None] * f
    c, s = amp * np.cos(a)[:, None], amp * np.sin(a)[:, None]
    i = np.arange(r)
    u, w = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
    y[..., u] = x[..., u] * c - x[..., w] * s
    y[..., w] = x[..., u] * s + x[..., w] * c
    return y
