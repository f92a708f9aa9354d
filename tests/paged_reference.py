"""The paged 4-bit cache in plain numpy and 64 bits: its format, its bookkeeping, the attention and the selection, written
from the formulas in include/lychee.h."""
import math

import numpy as np

D = 128
TILE, TILE_BYTES = 16, 2176
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def to_bf16_bits(x):
    """Round-to-nearest-even bf16 bits of finite float64 values that bf16 holds exactly or nearly."""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def from_bf16_bits(b):
    with np.errstate(invalid="ignore"):  # (NaN)
        return (np.asarray(b, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantise(x):
    """Codes [n, 128] and scale bytes [n, 4] of float64 rows."""
    g = np.asarray(x, np.float64).reshape(-1, 4, 32)
    codes = np.zeros(g.shape, np.uint8)
    scales = np.zeros(g.shape[:2], np.uint8)
    for i in range(g.shape[0]):
        for j in range(4):
            v = g[i, j]
            if not np.isfinite(v).all():
                scales[i, j] = 255
                continue
            big = np.abs(v).max()
            e = -125
            if big > 0:
                e = max(-125, min(125, math.ceil(math.log2(big / 6.0)) - 1))
                while e < 125 and big > 6.0 * 2.0 ** e:
                    e += 1
            scales[i, j] = e + 127
            u = np.abs(v) / 2.0 ** e
            d = np.abs(u[:, None] - GRID[:8])
            near = d == d.min(1, keepdims=True)
            pick = np.where(near.sum(1) == 1, near.argmax(1), 0)
            for t in np.nonzero(near.sum(1) == 2)[0]:  # (a tie: the even code)
                pick[t] = [c for c in np.nonzero(near[t])[0] if c % 2 == 0][0]
            codes[i, j] = pick + 8 * np.signbit(v)
    return codes.reshape(-1, D), scales


def dequantise(codes, scales):
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (GRID[codes].reshape(-1, 4, 32) * s[:, :, None]).reshape(-1, D)


class Cache:
    """The bytes of a layer's cache, as lychee.h lays them out."""

    def __init__(self, n_pages, page, heads, page_tiles=0, fill=0):
        self.page, self.heads = page, heads
        self.page_tiles = page_tiles or heads * page // TILE
        self.bytes = np.full((n_pages * self.page_tiles, TILE_BYTES), fill, np.uint8)

    def _at(self, slot, head):
        p, off = divmod(int(slot), self.page)
        return p * self.page_tiles + head * (self.page // TILE) + off // TILE, off % TILE

    def write(self, slot, head, k, v):
        """Codes and scales (quantise) of one token's key and value."""
        t, r = self._at(slot, head)
        for i, (codes, scales) in enumerate((k, v)):
            self.bytes[t, r * 128 + 64 * i:r * 128 + 64 * i + 64] = codes[0::2] | (codes[1::2] << 4)
            self.bytes[t, 2048 + np.arange(4 * i, 4 * i + 4) * 16 + r] = scales

    def rows(self, slots, head):
        """K and V [n, 128] of tokens, in 64 bits; a negative slot has zeros."""
        out = np.zeros((2, len(slots), D))
        for n, s in enumerate(slots):
            if s < 0:
                continue
            t, r = self._at(s, head)
            for i in range(2):
                b = self.bytes[t, r * 128 + 64 * i:r * 128 + 64 * i + 64]
                codes = np.empty(D, np.uint8)
                codes[0::2], codes[1::2] = b & 15, b >> 4
                out[i, n] = dequantise(codes[None], self.bytes[t, 2048 + np.arange(4 * i, 4 * i + 4) * 16 + r][None])[0]
        return out


def slots_of(table_row, n, page, n_pages):
    """Slots of a request's first n tokens; -1 where the table names no page."""
    t = np.arange(n)
    p = np.asarray(table_row)[t // page].astype(np.int64)
    return np.where((p >= 0) & (p < n_pages), p * page + t % page, -1)


class Pool:
    """lychee_release_pages and lychee_plan_pages, one request and one token at a time."""

    def __init__(self, free, page, max_pages, n_pages):
        self.free, self.page, self.max_pages, self.n_pages = list(free), page, max_pages, n_pages

    def release(self, done, lengths, table):
        for b, d in enumerate(done):
            if d:
                for e in range(-(-int(lengths[b]) // self.page)):
                    self.free.append(int(table[b, e]))
                lengths[b] = 0

    def plan(self, lengths, new, table, n_slots):
        """(status, slots, token_start); lengths and table change in place."""
        B = len(lengths)
        fail = lambda s: (s, np.full(n_slots, -1), np.zeros(B + 1, np.int64))  # noqa: E731
        if any(l < 0 or n < 0 or l + n > self.max_pages * self.page for l, n in zip(lengths, new)):
            return fail(-1)
        if sum(new) > n_slots:
            return fail(-2)
        need = sum(-(-int(l + n) // self.page) - -(-int(l) // self.page) for l, n in zip(lengths, new))
        if need > len(self.free):
            return fail(need - len(self.free))
        slots, start = [], [0]
        for b in range(B):
            for t in range(int(lengths[b]), int(lengths[b] + new[b])):
                if t % self.page == 0:
                    table[b, t // self.page] = self.free.pop()
                p = int(table[b, t // self.page])
                slots.append(p * self.page + t % self.page if 0 <= p < self.n_pages else -1)
            lengths[b] += new[b]
            start.append(len(slots))
        return 0, np.array(slots + [-1] * (n_slots - len(slots))), np.array(start)


def attend(q, k, v):
    """Outputs [G, 128], what they may be off by, and the logits [G, n] with theirs, of queries on n rows.

    Errors.  A logit is a sum of 128 products of exact operands in 32 bits: off by at most 130 * 2^-24 of the sum of the
    products' magnitudes, and by 2^-22 of itself for the scale; a weight 2^s is off by the logit's error, by the rounding of
    its exponent (|s| log2 e 2^-24 and the maximum's), by 2^-22 for the exponential and 2^-16 as the sum of two bf16 numbers.
    The sums over n tokens add n/16 * 2^-24 (sixteen lanes and more share them) and as much again where partials are merged.
    Numerator and denominator carry that error once each.  Last, the output is rounded to bf16: 2^-8 of it."""
    n = len(k)
    if n == 0:
        return np.zeros((len(q), D)), np.zeros((len(q), D)), np.zeros((len(q), 0)), np.zeros((len(q), 0))
    s = q @ k.T / math.sqrt(D)
    off = (np.abs(q) @ np.abs(k).T / math.sqrt(D)) * 130 * 2.0 ** -24 + np.abs(s) * 2.0 ** -22
    w = np.exp(s - s.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    each = off.max(1) * 2 + np.abs(s).max(1) * 4 * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -16 + (n / 8 + 64) * 2.0 ** -24
    o = w @ v
    return o, 2.0 ** -8 * np.abs(o) + 2 * each[:, None] * (w @ np.abs(v)), s, off


def top(scores, k):
    """Eq. 2 on one row: the k highest positions, ties to the lower, ascending; NaN as -infinity."""
    x = np.where(np.isnan(scores), -np.inf, np.asarray(scores, np.float64))
    return np.sort(np.lexsort((np.arange(len(x)), -x))[:k])
