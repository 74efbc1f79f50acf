"""Plain 64-bit forms of the 4-bit KV cache, the attention mass and the
eviction of tokens (include/recguide.h), in numpy, one element or token at a
time where that is clearest.  Written from the definitions; nothing of the
library is used."""
from __future__ import annotations

from typing import List, Optional, Tuple

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
PAGE = 16


def bf16_values(bits: np.ndarray) -> np.ndarray:
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def encode(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """4-bit codes [.., D] and scale bytes [.., D/32] of rows x [.., D] in float64.
    Groups with an infinity or a NaN get scale byte 255; their codes say nothing."""
    groups = x.reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(groups).all(axis=-1)
    groups = np.where(finite[..., None], groups, 0.0)
    top = np.abs(groups).max(axis=-1)
    frac, e = np.frexp(top)  # top = frac 2^e, 0.5 <= frac < 1: power of two 2^(e-1), mantissa 2 frac
    b = np.clip(np.where(top > 0, e - 1 + 127 + (2 * frac >= 1.75) - 2, 1), 1, 252).astype(np.int64)
    y = np.abs(groups) / np.exp2(b.astype(np.float64) - 127)[..., None]
    # nearest of the grid, ties to the even code
    dist = np.abs(np.minimum(y, 6.0)[..., None] - GRID)
    best = dist.min(axis=-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), near.argmax(axis=-1))
    code = code + 8 * np.signbit(groups)
    return code.reshape(x.shape).astype(np.int64), np.where(finite, b, 255)


def decode(code: np.ndarray, b: np.ndarray) -> np.ndarray:
    v = GRID[code & 7] * np.where(code >= 8, -1.0, 1.0)
    v = v.reshape(*b.shape, 32) * np.where(b == 255, np.nan, np.exp2(b.astype(np.float64) - 127))[..., None]
    return v.reshape(code.shape)


def _code_places(D: int, kv: int) -> np.ndarray:
    """Byte of a block that holds code byte i of slot s: [16, D/2]."""
    half = 8 * D + D // 2
    s, i = np.meshgrid(np.arange(16), np.arange(D // 2), indexing="ij")
    if kv == 0:
        return (i // 32) * 512 + s * 32 + i % 32
    vb = D // 64
    return half + (((s // 8) * 32 + i // vb) * 8 + s % 8) * vb + i % vb


def _scale_places(D: int, kv: int) -> np.ndarray:
    """Byte of a block that holds scale g of slot s: [16, D/32]."""
    half = 8 * D + D // 2
    s, g = np.meshgrid(np.arange(16), np.arange(D // 32), indexing="ij")
    if kv == 0:
        return 8 * D + s * (D // 32) + g
    return half + 8 * D + ((s // 8) * (D // 32) + g) * 8 + s % 8


def write_token(pool: np.ndarray, page: int, head: int, slot: int, kv: int, x: np.ndarray) -> None:
    """Row x [D] as K (kv 0) or V (1) of one token of a pool [pages, Hkv, 17 D] of bytes."""
    D = x.shape[-1]
    code, b = encode(x)
    pool[page, head, _code_places(D, kv)[slot]] = code[0::2] + 16 * code[1::2]
    pool[page, head, _scale_places(D, kv)[slot]] = b


def read_page(pool: np.ndarray, page, head: int, kv: int) -> np.ndarray:
    """Values [16, D] (or [n, 16, D] for several pages)."""
    D = pool.shape[-1] // 17
    block = pool[page, head]
    byte = block[..., _code_places(D, kv)].astype(np.int64)
    code = np.stack([byte & 15, byte >> 4], axis=-1).reshape(*byte.shape[:-1], D)
    return decode(code, block[..., _scale_places(D, kv)].astype(np.int64))


def tokens(pool: np.ndarray, pages: np.ndarray, head: int, T: int, kv: int) -> np.ndarray:
    D = pool.shape[-1] // 17
    return read_page(pool, pages, head, kv).reshape(-1, D)[:T]


def visible(L: int, V: int, n: int, branches=None) -> np.ndarray:
    """Mask [n, L + n]: Eq. 1, per branch where a list of (prefix, lead, rows) is given."""
    see = np.zeros((n, L + n), dtype=bool)
    for i in range(V):
        see[i, :L + i + 1] = True
    at = V
    for prefix, lead, rows in (branches if branches else ([(V, 0, n - V)] if n > V else [])):
        for t in range(rows):
            see[at + t, :L + prefix] = True
            see[at + t, L + at:L + at + (t + 1 if t < lead else rows)] = True
        at += rows
    return see


def attention(q: np.ndarray, K: np.ndarray, V: np.ndarray, see: np.ndarray, scale: float):
    """One request and KV head: q [n, g, D], K and V [T, D] -> out [n, g, D],
    lse [n, g], and the mean of |v| under the same weights (an error bound's scale)."""
    s = np.einsum("ngd,td->ngt", q, K) * scale
    s = np.where(see[:, None, :], s, -np.inf)
    top = s.max(axis=-1, keepdims=True)
    p = np.exp(s - top)
    z = p.sum(axis=-1, keepdims=True)
    Vs = np.where(see.any(axis=0)[:, None], V, 0.0)
    return (p / z) @ Vs, (top + np.log(z))[..., 0], (p / z) @ np.abs(Vs)


def mass(old: np.ndarray, q: np.ndarray, K: np.ndarray, lse: np.ndarray, L: int, V: int, count: Optional[int],
         decay: float, scale: float) -> np.ndarray:
    """One request and KV head: old and result [L + V]; q [n, g, D], lse [n, g]."""
    w = np.zeros(L + V)
    for i in range(min(max(V if count is None else count, 0), V)):
        j = np.arange(L + i + 1)
        w[j] += np.exp(q[i] @ K[j].T * scale - lse[i][:, None]).sum(axis=0)
    hist = np.zeros(L + V)
    if decay != 0:
        hist[:L] = decay * old[:L]
    return hist + w


def evict(score: np.ndarray, positions: np.ndarray, keep: int, sink: int, recent: int,
          total: int) -> List[Tuple[int, int]]:
    """Moves (to, from) of one request and KV head: score and positions [L] of
    its slots, `total` the positions its whole sequence has had."""
    L = len(score)
    keep = min(keep, L)
    if keep == 0:
        return []
    safe = (positions < sink) | (positions >= total - recent)
    # protected first, then larger scores, then lower slots
    order = sorted(range(L), key=lambda j: (0 if safe[j] else 1, 0.0 if safe[j] else -float(score[j]), j))
    kept = np.zeros(L, dtype=bool)
    kept[order[:keep]] = True
    holes = [j for j in range(keep) if not kept[j]]
    movers = [j for j in range(keep, L) if kept[j]]
    return list(zip(holes, movers))
