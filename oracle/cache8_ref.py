"""Plain fp64 reference of the 8-bit cache, of what its attention gathers and of its eviction
(test infrastructure only).

The format (include/stepkv_cache8.h): e4m3 numbers times a power of two that the 64 tokens of a
block share. One ``Head8`` is one (layer, KV head, sequence): its tokens in the order of their
rows, changed by the calls' definitions one token or block at a time, without streaming; floating
point is fp64 throughout.
"""
from __future__ import annotations

import numpy as np

__all__ = ["NUMBERS", "round8", "need", "Head8", "stay"]

BLOCK = 64
LEAST, MOST = -117, 119


def _numbers() -> np.ndarray:
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = np.nan if c & 127 == 127 else (-x if c & 128 else x)
    return out


NUMBERS = _numbers()  # by code
_GRID = NUMBERS[:127]  # the magnitudes, ascending; their codes are 0 .. 126


def round8(y: np.ndarray) -> np.ndarray:
    """Elements rounded to the nearest e4m3 number, ties to the even code, at most 448; NaN for
    what is not finite. (Signs of zeros are not kept apart.)"""
    a = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    hi = np.clip(np.searchsorted(_GRID, a), 1, 126)
    lo = hi - 1
    up, down = _GRID[hi] - a, a - _GRID[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isfinite(y), np.sign(y) * _GRID[code], np.nan)


def need(x: np.ndarray) -> int:
    """The exponent that some rows need together: the smallest e with max|x| <= 464 * 2^e."""
    fin = np.abs(x[np.isfinite(x)])
    top = fin.max() if fin.size else 0.0
    for e in range(LEAST, MOST):
        if top <= 464.0 * 2.0 ** e:
            return e
    return MOST


def stay(weights, positions, keep: int, first: int, recent: int, seen: int) -> np.ndarray:
    """Which tokens stay, as a mask: those that stay in any case (the lower rows first), then by
    weight, the greatest first (NaN as -inf, equal ones by row)."""
    w = np.where(np.isnan(weights), -np.inf, np.asarray(weights, np.float64))
    always = (positions < first) | (positions >= seen - recent)
    order = sorted(range(len(w)), key=lambda j: (not always[j], 0.0 if always[j] else -w[j], j))
    mask = np.zeros(len(w), bool)
    mask[order[:keep]] = True
    return mask


class Head8:
    """The tokens of one head of one sequence."""

    def __init__(self, d: int):
        self.num = [np.zeros((0, d)), np.zeros((0, d))]  # elements of K and V
        self.exp = [[], []]                              # exponents of their blocks
        self.weights, self.positions = np.zeros(0), np.zeros(0, np.int64)

    def __len__(self):
        return len(self.weights)

    def values(self, which: int) -> np.ndarray:
        e = np.repeat(np.array(self.exp[which], np.float64), BLOCK)[:len(self)]
        return self.num[which] * 2.0 ** e[:, None]

    def append(self, k, v, positions, weights=None):
        """New tokens (fp64 rows), in one call."""
        n, m = len(self), len(k)
        for which, x in enumerate((k, v)):
            num = np.concatenate([self.num[which], np.zeros_like(x)])
            for b in range(n // BLOCK, -(-(n + m) // BLOCK) if m else 0):
                lo, hi = max(n, b * BLOCK), min(n + m, (b + 1) * BLOCK)
                new = x[lo - n:hi - n]
                if lo == b * BLOCK:
                    self.exp[which].append(need(new))
                else:
                    self._grow(which, num, b, lo, need(new))
                num[lo:hi] = round8(new / 2.0 ** self.exp[which][b])
            self.num[which] = num
        self.weights = np.concatenate([self.weights, np.zeros(m) if weights is None else weights])
        self.positions = np.concatenate([self.positions, positions])

    def _grow(self, which, num, b, end, e):
        """Block b, tokens up to `end`, takes exponent e if it is greater than its own."""
        old = self.exp[which][b]
        if e > old:
            rows = slice(b * BLOCK, min(end, (b + 1) * BLOCK))
            num[rows] = round8(num[rows] * 2.0 ** (old - e))
            self.exp[which][b] = e

    def evict(self, keep: int, first: int, recent: int, seen: int):
        n = len(self)
        if n <= keep:
            return
        mask = stay(self.weights, self.positions, keep, first, recent, seen)
        to, frm = np.nonzero(~mask[:keep])[0], keep + np.nonzero(mask[keep:])[0]
        assert len(to) == len(frm)
        for which in (0, 1):
            x = self.values(which)[frm]
            num = self.num[which][:keep].copy()
            for b in sorted(set(to // BLOCK)):
                into = to // BLOCK == b
                self._grow(which, num, b, keep, need(x[into]) if into.any() else LEAST)
            num[to] = round8(x / 2.0 ** np.array(self.exp[which])[to // BLOCK][:, None]) if len(to) else num[to]
            self.num[which] = num
            self.exp[which] = self.exp[which][:-(-keep // BLOCK)]
        self.weights[to], self.positions[to] = self.weights[frm], self.positions[frm]
        self.weights, self.positions = self.weights[:keep].copy(), self.positions[:keep].copy()
