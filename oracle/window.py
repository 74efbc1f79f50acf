"""Plain 64-bit forms of rotated appends, the 8-bit KV cache and attention over
a window (include/recguide.h), in numpy.  Written from the definitions; nothing
of the library is used."""
from __future__ import annotations

import math
from typing import Optional, Tuple

import numpy as np

PAGE = 16
# The 256 e4m3 numbers: sign, 4 exponent bits of bias 7, 3 mantissa bits, 0x7f NaN.
GRID = np.array([math.nan if c == 127 else
                 (c % 8) * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(128)])
GRID = np.concatenate([GRID, -GRID])


def rotate(x: np.ndarray, position: np.ndarray, inv_freq: np.ndarray, interleaved: bool) -> np.ndarray:
    """Rows x [rows, heads, D] turned by their positions.  The angle is the product
    in 64 bits: exact for fp32 frequencies and positions below 2^29."""
    y = x.copy()
    half = len(inv_freq)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        w = (position.astype(np.float64) * np.float64(inv_freq[j]))[:, None]
        y[..., a] = x[..., a] * np.cos(w) - x[..., b] * np.sin(w)
        y[..., b] = x[..., b] * np.cos(w) + x[..., a] * np.sin(w)
    return y


def turns(position: np.ndarray, inv_freq: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """Cosine and sine [rows, dims / 2] of the exact angles of fp32 frequencies, in
    80 bits: a position below 2^31 times 24 bits needs 55, of which 64 bits hold 53."""
    assert inv_freq.dtype == np.float32 and np.finfo(np.longdouble).nmant >= 63
    w = position.astype(np.longdouble)[:, None] * inv_freq.astype(np.longdouble)
    return np.cos(w), np.sin(w)


def exponent(top: float) -> int:
    """Exponent of the scale for a largest magnitude."""
    if top == 0:
        return -117
    frac, e = math.frexp(top)
    return min(max(e - 1 + (2 * frac >= 1.75) - 8, -117), 119)


def codes(x: np.ndarray, scale: float) -> np.ndarray:
    """Bytes of values at a scale: the nearest number, ties to the even code."""
    y = np.where(np.isfinite(x), x, 0.0) / scale
    mag = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(GRID[:127], mag, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - mag, mag - GRID[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isfinite(x), c + 128 * np.signbit(y), 127).astype(np.uint8)


def place(D: int, kv: int) -> np.ndarray:
    """Byte of a block that holds element d of slot s: [16, D]."""
    s, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    if kv == 0:
        return (d // 32) * 512 + s * 32 + d % 32
    return 16 * D + ((s // 8) * D + d) * 8 + s % 8


def values(pool: np.ndarray, scales: np.ndarray, page, head: int, kv: int) -> np.ndarray:
    """Values [16, D] of a page (or [n, 16, D] of several)."""
    D = pool.shape[-1] // 32
    s = np.asarray(scales[page, head, kv], dtype=np.float64)
    return GRID[pool[page, head][..., place(D, kv)]] * s[..., None, None]


def append8(pool: np.ndarray, scales: np.ndarray, pages: np.ndarray, L: int, x: np.ndarray, kv: int) -> None:
    """Rows x [n, Hkv, D] of one request as its tokens L, L + 1, ..., in place."""
    n, hkv, D = x.shape
    at = place(D, kv)
    for p in range(L // PAGE, (L + n - 1) // PAGE + 1 if n else 0):
        s0, s1 = max(L - p * PAGE, 0), min(L + n - p * PAGE, PAGE)
        for h in range(hkv):
            new = x[p * PAGE + s0 - L:p * PAGE + s1 - L, h]
            top = np.abs(new[np.isfinite(new)]).max(initial=0.0)
            scale = 2.0 ** exponent(top)
            block = pool[pages[p], h]
            if s0 > 0:
                old = values(pool, scales, pages[p], h, kv)[:s0]
                scale = max(scale, float(scales[pages[p], h, kv]))
                block[at[:s0]] = codes(old, scale)
            block[at[s0:s1]] = codes(new, scale)
            scales[pages[p], h, kv] = scale


def visible(L: int, V: int, n: int, branches=None, size: Optional[int] = None, sink: int = 0) -> np.ndarray:
    """Mask [n, L + n]: Eq. 1, per branch where a list of (prefix, lead, rows) is
    given; with a window, of the keys outside a row's own draft block or branch
    those of the latest `size` positions up to its own, and of positions below `sink`."""
    size = 1 << 60 if size is None else size
    see = np.zeros((n, L + n), dtype=bool)

    def near(t, p):
        return t < sink or t > p - size

    for i in range(V):
        for t in range(L + i + 1):
            see[i, t] = near(t, L + i)
    at = V
    for prefix, lead, rows in (branches if branches else ([(V, 0, n - V)] if n > V else [])):
        for k in range(rows):
            for t in range(L + prefix):
                see[at + k, t] = near(t, L + prefix + k)
            see[at + k, L + at:L + at + (k + 1 if k < lead else rows)] = True
        at += rows
    return see
