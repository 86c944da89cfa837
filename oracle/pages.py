"""The paged 4-bit cache in NumPy float64 and sequential Python.

TEST INFRASTRUCTURE ONLY (see the package docstring).

A row of d channels is held as four-bit floats E2M1 (sign, two exponent bits of
bias 1, one mantissa bit) with one power of two per 32 channels.  The power is
the one under which the block's largest element is off by least: 2^(e-2) for a
largest magnitude in [2^e, 1.75 * 2^e), 2^(e-1) from there to 2^(e+1), kept
within 2^-125 .. 2^125.  Elements go to the nearest value, ties to the even
code.  A block that holds a NaN or an infinity becomes 32 NaN.

The bookkeeping (``PageBook``) takes the entries of a call one by one, which is
what the device calls promise.
"""

from __future__ import annotations

import math

import numpy as np

__all__ = ["E2M1", "NAN_SCALE", "mx4_quantise", "mx4_values", "mx4_round", "page_bytes", "page_pack", "page_unpack",
           "PageBook"]

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_SCALE = 255


def mx4_quantise(x: np.ndarray):
    """(codes uint8 [..., d], scale bytes uint8 [..., d / 32]) of rows x [..., d]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    bad = ~np.isfinite(blocks).all(axis=-1)
    b = np.where(bad[..., None], 0.0, blocks)
    m = np.abs(b).max(axis=-1)
    mant, e = np.frexp(m)                      # m = mant * 2^e with mant in [0.5, 1)
    e = e - 1 + (mant >= 0.875)
    s = np.clip(np.where(m > 0, e + 125, 0), 2, 252)
    y = np.abs(b) / np.exp2(s - 127.0)[..., None]
    # nearest of the eight magnitudes; of two equally near ones the even code
    dist = np.abs(y[..., None] - E2M1)
    near = dist == dist.min(axis=-1, keepdims=True)
    code = np.where(near & (np.arange(8) % 2 == 0), np.arange(8), np.where(near, 8 + np.arange(8), 99)).min(axis=-1) % 8
    code = code + 8 * np.signbit(b)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, NAN_SCALE, s).astype(np.uint8)


def mx4_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """float64 rows [..., d] of codes [..., d] and scale bytes [..., d / 32]."""
    codes = np.asarray(codes)
    v = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes % 8]
    v = v.reshape(codes.shape[:-1] + (codes.shape[-1] // 32, 32))
    s = np.asarray(scales, dtype=np.float64)
    unit = np.where(s == NAN_SCALE, np.nan, np.exp2(np.where(s == NAN_SCALE, 0.0, s - 127.0)))
    return (v * unit[..., None]).reshape(codes.shape)


def mx4_round(x: np.ndarray) -> np.ndarray:
    """The float64 values that rows x are held as."""
    return mx4_values(*mx4_quantise(x))


def page_bytes(page: int, d: int) -> int:
    return page * d + 2 * page * (d // 32)


def page_pack(k: np.ndarray, v: np.ndarray) -> np.ndarray:
    """uint8 [..., page bytes] blocks of key and value rows [..., page, d]."""
    lead = k.shape[:-2]
    codes, scales = [], []
    for x in (k, v):
        c, s = mx4_quantise(x)
        codes.append((c[..., 0::2] | (c[..., 1::2] << 4)).reshape(lead + (-1,)))
        scales.append(np.swapaxes(s, -1, -2).reshape(lead + (-1,)))
    return np.concatenate(codes + scales, axis=-1)


def page_unpack(block: np.ndarray, page: int, d: int):
    """(keys, values) float64 [..., page, d] of page blocks."""
    lead = block.shape[:-1]
    half, ns = page * d // 2, page * (d // 32)
    out = []
    for i in (0, 1):
        p = block[..., i * half:(i + 1) * half].reshape(lead + (page, d // 2))
        c = np.stack([p & 15, p >> 4], axis=-1).reshape(lead + (page, d))
        s = block[..., 2 * half + i * ns:2 * half + (i + 1) * ns].reshape(lead + (d // 32, page))
        out.append(mx4_values(c, np.swapaxes(s, -1, -2)))
    return tuple(out)


class PageBook:
    """refs, table, held and length of a pool (int64 arrays), entry by entry."""

    def __init__(self, refs, table, held, length, page: int):
        self.refs, self.table, self.held, self.length = (np.array(x, dtype=np.int64) for x in (refs, table, held, length))
        self.page = page
        self.S, self.M = self.table.shape
        self.n_pages = len(self.refs)

    def _take(self, free: list, left: int, need: int):
        """The next `need` pages of the ascending list `free`, of which `left` are not spoken for
        (negative once an entry could not be served: no later one that needs a page is)."""
        return None if need > max(left, 0) else [free.pop(0) for _ in range(need)]

    def extend(self, seq, add):
        """(start list, missing pages)."""
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        left, total, F = len(free), 0, len(free)
        start, seen = [], set()
        for slot, a in zip(seq, add):
            if not 0 <= slot < self.S or slot in seen:
                start.append(-1)
                continue
            seen.add(slot)
            if a < 0 or self.length[slot] + a > self.M * self.page:
                start.append(-1)
                continue
            need = max(0, math.ceil((self.length[slot] + a) / self.page) - self.held[slot])
            got = self._take(free, left, need)
            left -= need
            total += need
            if got is None:
                start.append(-1)
                continue
            for p in got:
                self.table[slot, self.held[slot]] = p
                self.refs[p] = 1
                self.held[slot] += 1
            start.append(int(self.length[slot]))
            self.length[slot] += a
        return start, max(0, total - F)

    def fork(self, src, dst):
        """(done list, missing pages, copies): copies lists (source page, fresh page, rows)."""
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        left, total, F = len(free), 0, len(free)
        held0, length0, table0 = self.held.copy(), self.length.copy(), self.table.copy()
        done, copies, seen = [], [], set()
        for a, b in zip(src, dst):
            first = b not in seen
            seen.add(b)
            if not (first and 0 <= a < self.S and 0 <= b < self.S):
                done.append(0)
                continue
            if held0[b] != 0 or length0[b] != 0:
                done.append(0)
                continue
            full, rest = divmod(int(length0[a]), self.page)
            last = int(table0[a, full]) if rest else -1
            need = 1 if 0 <= last < self.n_pages else 0      # a page that is not there is passed on as such
            got = self._take(free, left, need)
            left -= need
            total += need
            if got is None:
                done.append(0)
                continue
            for i in range(full):
                self.table[b, i] = table0[a, i]
                if 0 <= table0[a, i] < self.n_pages:
                    self.refs[table0[a, i]] += 1
            if rest:
                self.table[b, full] = got[0] if need else last
            if need:
                self.refs[got[0]] = 1
                copies.append((last, got[0], rest))
            self.held[b], self.length[b] = full + (rest > 0), length0[a]
            done.append(1)
        return done, max(0, total - F), copies

    def free(self, seq):
        for slot in seq:
            if 0 <= slot < self.S:
                for i in range(self.held[slot]):
                    if 0 <= self.table[slot, i] < self.n_pages:
                        self.refs[self.table[slot, i]] -= 1
                self.held[slot] = self.length[slot] = 0
