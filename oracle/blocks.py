"""The paged 8-bit cache in NumPy float64 and sequential Python.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A block is ``page`` tokens of one layer and KV head: eight-bit floats E4M3 (a sign,
four exponent bits of bias 7, three of mantissa; no infinities) times one power of
two for its keys and one for its values.  ``BlockRows`` holds a sequence's blocks as
code values (not bytes) and takes writes one call at a time, which is what the
device calls promise; rotation, block scores and attention are their formulas.
"""

from __future__ import annotations

import math

import numpy as np

__all__ = ["E4M3", "e4m3_round", "e4m3_values", "e4m3_codes", "block_scale", "block_bytes", "block_unpack", "BlockRows",
           "rotate", "round_to", "block_scores", "top_blocks", "rows_seen", "attend"]

# the magnitudes of codes 0 .. 126
E4M3 = np.array([f / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + f / 8.0) * 2.0 ** (e - 7)
                 for e in range(16) for f in range(8)][:127])
SCALE_MIN, SCALE_MAX = 27, 246


def e4m3_round(y: np.ndarray) -> np.ndarray:
    """The nearest E4M3 value of every element, of two equally near ones that of the even code; magnitudes above 448
    become 448, infinities and NaN become NaN."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    up = np.clip(np.searchsorted(E4M3, a, side="left"), 0, 126)      # first value >= a
    down = np.maximum(up - 1, 0)
    du, dd = E4M3[up] - a, a - E4M3[down]
    code = np.where(du < dd, up, np.where(dd < du, down, np.where(up % 2 == 0, up, down)))
    return np.where(np.isfinite(y), np.copysign(E4M3[code], y), np.nan)


def e4m3_values(codes: np.ndarray) -> np.ndarray:
    """float64 values of code bytes."""
    codes = np.asarray(codes)
    mag = np.append(E4M3, np.nan)[codes & 127]
    return np.where(codes >= 128, -mag, mag)


def e4m3_codes(values: np.ndarray) -> np.ndarray:
    """Bytes of E4M3 values (NaN as 127)."""
    values = np.asarray(values, dtype=np.float64)
    code = np.searchsorted(E4M3, np.where(np.isnan(values), 0.0, np.abs(values)))
    return np.where(np.isnan(values), 127, code + 128 * np.signbit(values)).astype(np.uint8)


def block_scale(rows: np.ndarray) -> int:
    """Scale byte of new rows: the smallest s with every finite magnitude <= 448 * 2^(s - 127), within its limits."""
    a = np.abs(rows[np.isfinite(rows)])
    m = a.max() if a.size else 0.0
    s = SCALE_MIN
    while s < SCALE_MAX and m > 448.0 * 2.0 ** (s - 127):
        s += 1
    return s


def block_bytes(page: int, d: int) -> int:
    return 2 * page * d + 128 + 2 * d


def block_unpack(block: np.ndarray, page: int, d: int):
    """(key codes, value codes [..., page, d], scale bytes [..., 2], bound codes [..., 2, d]) of block bytes."""
    lead, n = block.shape[:-1], page * d
    return (block[..., :n].reshape(lead + (page, d)), block[..., n:2 * n].reshape(lead + (page, d)),
            block[..., 2 * n:2 * n + 2], block[..., 2 * n + 128:].reshape(lead + (2, d)))


class BlockRows:
    """The blocks of one sequence, layer and KV head."""

    def __init__(self, page: int, d: int, blocks: int):
        self.page, self.d = page, d
        self.code = np.full((2, blocks, page, d), np.nan)     # keys, values, in units of the scale
        self.s = np.zeros((2, blocks), dtype=np.int64)
        self.bound = np.full((2, blocks, d), np.nan)          # minima, maxima, in units of the key scale

    def write(self, start: int, k: np.ndarray, v: np.ndarray):
        """Rows k, v [n, d] into positions start .."""
        n, P = len(k), self.page
        for i in range(start // P, -(-(start + n) // P) if n else start // P):
            r0, r1 = max(start - i * P, 0), min(start + n - i * P, P)
            for x, rows in ((0, k), (1, v)):
                new = np.asarray(rows, dtype=np.float64)[i * P + r0 - start:i * P + r1 - start]
                s = block_scale(new)
                if r0:
                    old = self.s[x, i]
                    s = max(s, old)
                    self.code[x, i, :r0] = e4m3_round(self.code[x, i, :r0] * 2.0 ** (old - s))
                    if x == 0:
                        self.bound[:, i] = e4m3_round(self.bound[:, i] * 2.0 ** (old - s))
                self.s[x, i] = s
                codes = e4m3_round(new * 2.0 ** (127 - s))
                self.code[x, i, r0:r1] = codes
                if x == 0:
                    both = [codes.min(0), codes.max(0)]       # NaN wins
                    if r0:
                        both = [np.minimum(both[0], self.bound[0, i]), np.maximum(both[1], self.bound[1, i])]
                    self.bound[:, i] = both

    def values(self, n: int):
        """Key and value rows float64 [n, d]."""
        unit = 2.0 ** (self.s - 127.0)
        return tuple((self.code[x] * unit[x][:, None, None]).reshape(-1, self.d)[:n] for x in (0, 1))

    def bounds(self):
        """(minima, maxima) float64 [blocks, d]."""
        unit = 2.0 ** (self.s[0] - 127.0)
        return self.bound[0] * unit[:, None], self.bound[1] * unit[:, None]


def rotate(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, position: np.ndarray, pairs: bool) -> np.ndarray:
    """float64 rows x [..., T, d] at positions [T], the first 2 cos.shape[1] channels turned; NaN without a position."""
    x = np.asarray(x, dtype=np.float64)
    half = cos.shape[1]
    a = np.arange(half) * 2 if pairs else np.arange(half)
    b = a + 1 if pairs else a + half
    ok = (position >= 0) & (position < cos.shape[0])
    at = np.where(ok, position, 0)
    c, s = cos[at].astype(np.float64), sin[at].astype(np.float64)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    y[..., ~ok, :] = np.nan
    return y


def round_to(y: np.ndarray, bits: int) -> np.ndarray:
    """Normal numbers y rounded once to `bits` significant bits, ties to even."""
    m, e = np.frexp(np.asarray(y, dtype=np.float64))
    return np.ldexp(np.round(np.ldexp(m, bits)), e - bits)


def rows_seen(length: int, T: int, t: int, max_tokens: int, start: int | None = None) -> int:
    """Rows that query token t of T sees."""
    if start is not None and start < 0:
        return 0
    start = length - T if start is None else start
    return max(0, min(start + t + 1, length, max_tokens))


def block_scores(q: np.ndarray, lo: np.ndarray, hi: np.ndarray) -> np.ndarray:
    """Scores float32 [blocks] of the query heads q [G, d]: the sum over heads and channels of max(q, 0) hi + min(q, 0) lo,
    from which no key of a block can give a higher sum of products; a NaN bound makes a NaN score."""
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.zeros(len(lo))
        for h in range(len(q)):
            x += (np.maximum(q[h], 0) * hi + np.minimum(q[h], 0) * lo).sum(-1)
        return x.astype(np.float32)


def top_blocks(score: np.ndarray, k: int, first: int, last: int, missing=()) -> list:
    """Indices, ascending, of the first `first`, the last `last` and the highest of the rest, k in all, then -1."""
    n = len(score)

    def rank(i):
        if i < first or i >= n - last:
            return (0, 0.0, i)
        if i in missing or math.isnan(score[i]):
            return (2, 0.0, i)
        return (1, -float(score[i]), i)
    out = sorted(sorted(range(n), key=rank)[:k])
    return out + [-1] * (k - len(out))


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """(output [G, d], sum of p |v| [G, d], largest scale sum |q k|) of q [G, d] over rows k, v [n, d], float64."""
    if len(k) == 0:
        return np.zeros_like(q), np.zeros_like(q), 0.0
    x = scale * (q @ k.T)
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, p @ np.abs(v), float((scale * (np.abs(q) @ np.abs(k).T)).max())
