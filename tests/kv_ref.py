"""Plain implementation of the 4-bit key/value cache in NumPy, from the definitions in include/tpq.h: the quantiser in binary32
operation for operation, everything else in 64 bits."""
from __future__ import annotations

import numpy as np

BLOCK = 16


def bf16(x: np.ndarray) -> np.ndarray:
    """float32 -> BF16 patterns, round to nearest even; NaN -> 0x7FC0."""
    x = np.ascontiguousarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def wide(b: np.ndarray) -> np.ndarray:
    return (np.ascontiguousarray(b).astype(np.uint32) << 16).view(np.float32)


def quantise(x: np.ndarray):
    """x [..., dim] float32 -> codes (uint8), words (uint32)."""
    x = np.ascontiguousarray(x, np.float32)
    f = np.float32
    with np.errstate(all="ignore"):
        lo, hi, top = x.min(-1), x.max(-1), np.abs(x).max(-1)
        low = wide(bf16(lo))
        d = hi - low
        step = wide(bf16(np.maximum(np.maximum(d * f(1.0 / 15.0), top * f(2.0 ** -16)), f(2.0 ** -60))))
        bad = ~(d < np.inf) | ~np.isfinite(low)
        u = (x - low[..., None]) / step[..., None]
        codes = np.clip(np.rint(np.where(np.isfinite(u), u, 0)), 0, 15)
    codes = np.where(bad[..., None], 0, codes).astype(np.uint8)
    words = bf16(np.where(bad, f(1), step)).astype(np.uint32) | (np.where(bad, np.uint16(0x7FC0), bf16(low)).astype(np.uint32) << 16)
    return codes, words


def rotate(x: np.ndarray, table: np.ndarray, pos: np.ndarray, rot: int, interleaved: bool) -> np.ndarray:
    """x [rows, heads, dim] float32, binary32 with every product and sum rounded."""
    x = np.array(x, np.float32)
    cos, sin = table[pos, None, : rot // 2].astype(np.float32), table[pos, None, rot // 2: rot].astype(np.float32)
    ia, ib = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
    with np.errstate(all="ignore"):
        a, b = x[..., ia], x[..., ib]
        y = x.copy()
        y[..., ia], y[..., ib] = a * cos - b * sin, b * cos + a * sin
    return y


class Cache:
    """Pages as bytes, [pages][heads][page_size/16][block]."""

    def __init__(self, n_pages, heads, dim, page, fill=None, rng=None):
        self.heads, self.dim, self.page, self.n_pages = heads, dim, page, n_pages
        shape = (n_pages, heads, page // BLOCK, BLOCK * (dim + 8))
        self.bytes = rng.integers(0, 256, shape, dtype=np.uint8) if fill is None else np.full(shape, fill, np.uint8)

    def put(self, page, head, at, which, codes, word):
        half, b = self.dim // 2, self.bytes[page, head, at // BLOCK]
        r = at % BLOCK
        b[which * BLOCK * half + r * half:][:half] = codes[0::2] | (codes[1::2] << 4)
        b[2 * BLOCK * half + which * 4 * BLOCK + 4 * r:][:4] = np.frombuffer(np.uint32(word).tobytes(), np.uint8)

    def get(self, page, head, at, which):
        """(codes, word)"""
        half, b = self.dim // 2, self.bytes[page, head, at // BLOCK]
        r = at % BLOCK
        row = b[which * BLOCK * half + r * half:][:half]
        codes = np.empty(self.dim, np.uint8)
        codes[0::2], codes[1::2] = row & 15, row >> 4
        return codes, int.from_bytes(b[2 * BLOCK * half + which * 4 * BLOCK + 4 * r:][:4].tobytes(), "little")

    def sequence(self, table_row, length, head, which):
        """step [length], low [length], codes [length, dim], all float64; pages outside the pool: NaN steps."""
        pos = np.arange(length)
        page = np.asarray(table_row)[pos // self.page].astype(np.int64)
        ok = (page >= 0) & (page < self.n_pages)
        half, r = self.dim // 2, pos % BLOCK
        b = self.bytes[np.where(ok, page, 0), head, pos % self.page // BLOCK]
        i = np.arange(length)[:, None]
        row = b[i, which * BLOCK * half + r[:, None] * half + np.arange(half)]
        word = np.ascontiguousarray(b[i, 2 * BLOCK * half + which * 4 * BLOCK + 4 * r[:, None] + np.arange(4)]).view(np.uint32)[:, 0]
        codes = np.empty((length, self.dim))
        codes[:, 0::2], codes[:, 1::2] = row & 15, row >> 4
        return wide((word & 0xFFFF).astype(np.uint16)).astype(np.float64), wide((word >> 16).astype(np.uint16)).astype(np.float64), codes, ok


def append(cache, table, start, lengths, k, v, q=None, rot_table=None, rot=0, interleaved=False, positions=None):
    """Writes the rows k, v ([rows, heads, dim] float32) into `cache`; returns q rotated (BF16 patterns; rows of nobody 0)."""
    out = None if q is None else np.zeros(q.shape, np.uint16)
    for s in range(len(lengths)):
        n = start[s + 1] - start[s]
        for i in range(n):
            row, pos = start[s] + i, lengths[s] - n + i
            p = pos if positions is None else positions[row]
            kr = rotate(k[row:row + 1], rot_table, np.array([p]), rot, interleaved)[0] if rot else k[row]
            if q is not None:
                out[row] = bf16(rotate(q[row:row + 1], rot_table, np.array([p]), rot, interleaved)[0])
            for which, x in ((0, kr), (1, v[row])):
                codes, words = quantise(x)
                for h in range(cache.heads):
                    cache.put(table[s][pos // cache.page], h, pos % cache.page, which, codes[h], words[h])
    return out


def attention(cache, table, start, lengths, q, scale, window=0, first=0):
    """(out, bound): out [rows, heads, dim] float64 (rows of nobody NaN); bound: sum of weight * largest magnitude a value of the
    vector's range may have, over the sum of weights, for tolerances."""
    rows, heads, dim = q.shape
    group = heads // cache.heads
    out, bound = np.full((rows, heads, dim), np.nan), np.full((rows, heads, 1), np.nan)
    for s in range(len(lengths)):
        n, ln = start[s + 1] - start[s], int(lengths[s])
        if n == 0:
            continue
        for kh in range(cache.heads):
            ks, kl, kc, ok = cache.sequence(table[s], ln, kh, 0)
            vs, vl, vc, _ = cache.sequence(table[s], ln, kh, 1)
            K, Vv = kl[:, None] + ks[:, None] * kc, vl[:, None] + vs[:, None] * vc
            big = np.maximum(np.abs(vl), np.abs(vl + 15 * vs))
            t = np.arange(ln)
            for i in range(n):
                p = ln - n + i
                see = (t <= p) & ok
                if window:
                    see &= (t > p - window) | (t < first)
                qq = q[start[s] + i, kh * group:(kh + 1) * group].astype(np.float64)
                sl = slice(kh * group, (kh + 1) * group)
                if not see.any():
                    out[start[s] + i, sl], bound[start[s] + i, sl] = 0, 0
                    continue
                z = scale * (qq @ K[see].T)
                w = np.exp(z - z.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[start[s] + i, sl] = w @ Vv[see]
                bound[start[s] + i, sl] = (w @ big[see])[:, None]
    return out, bound
