"""Plain fp64 reference of the 4-bit cache and of what reads it (test infrastructure only).

The format (include/stepkv_cache4.h): elements {0, .5, 1, 1.5, 2, 3, 4, 6} with a sign times
2^e, e shared by 32 channels of a row: the smallest integer with max|x| <= 7 * 2^e, clamped to
[-124, 125], held as the byte e + 127 (255: the group held a NaN or an infinity). Elements are
rounded to the nearest, ties to the even code. Every function restates its definition without
blocking or streaming; floating point is fp64 throughout.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["LEVELS", "quantise4", "dequantise4", "block_bounds", "block_scores", "select_blocks",
           "attend"]

BLOCK, GROUP = 64, 32
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise4(x: np.ndarray):
    """Codes uint8 [..][d/2] and scale bytes uint8 [..][d/32] of values [..][d]."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    top = np.abs(g).max(axis=-1)
    bad = ~np.isfinite(top)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.ceil(np.log2(safe / 7.0)).astype(np.int64)
    e += safe > 7.0 * 2.0 ** e          # a logarithm rounded the wrong way
    e -= safe <= 7.0 * 2.0 ** (e - 1.0)
    e = np.clip(np.where(top == 0, -124, e), -124, 125)
    y = np.where(bad[..., None], 0.0, g) / (2.0 ** e)[..., None]
    dist = np.abs(np.abs(y)[..., None] - LEVELS)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # argmin takes the first: even codes win ties
    code = order[np.argmin(dist[..., order], axis=-1)]
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(y)).reshape(x.shape).astype(np.uint8)
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte


def dequantise4(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values [..][d] that codes and scale bytes stand for."""
    c = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    v = np.where(c & 8, -1.0, 1.0) * LEVELS[c & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, axis=-1)


def block_bounds(k: np.ndarray) -> np.ndarray:
    """[blocks][2][d]: least and greatest key value per channel over each 64 tokens of k [n][d]
    (NaN where one is NaN)."""
    nb = -(-k.shape[0] // BLOCK)
    out = np.empty((nb, 2, k.shape[1]))
    for b in range(nb):
        x = k[b * BLOCK:(b + 1) * BLOCK]
        out[b, 0], out[b, 1] = x.min(axis=0), x.max(axis=0)
    return out


def block_scores(q: np.ndarray, bounds: np.ndarray) -> np.ndarray:
    """[blocks]: sum over the heads q [G][d] and channels of max(q kmin, q kmax)."""
    with np.errstate(invalid="ignore"):
        return np.maximum(q[:, None] * bounds[None, :, 0], q[:, None] * bounds[None, :, 1]).sum(axis=(0, 2))


def select_blocks(score: np.ndarray, n: int, first: int, last: int) -> np.ndarray:
    """The n blocks attended to, ascending, -1 past the last: the first and last ones, the others
    by (score descending, block ascending), NaN as -inf."""
    nb = score.shape[0]
    out = np.full(n, -1, np.int32)
    if nb <= n:
        out[:nb] = np.arange(nb)
        return out
    forced = [b for b in range(nb) if b < first or b >= nb - last]
    rest = np.arange(first, nb - last)
    s = np.where(np.isnan(score), -np.inf, score)[rest]
    rest = rest[np.argsort(-s, kind="stable")][:n - len(forced)]
    out[:] = np.sort(np.concatenate([np.array(forced, np.int64), rest]))
    return out


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """(out [d], lse, sum p |v| [d], max |scale q| . |k|) of one query over n tokens; the last two
    bound what rounding may change."""
    if k.shape[0] == 0:
        return np.zeros(v.shape[1]), -math.inf, np.zeros(v.shape[1]), 0.0
    z = scale * (k @ q)
    m = z.max()
    p = np.exp(z - m)
    total = p.sum()
    return (p / total) @ v, m + math.log(total) if total > 0 else math.nan, (p / total) @ np.abs(v), \
        float(abs(scale) * (np.abs(k) @ np.abs(q)).max())
