"""Plain CPU implementation of the paged cache of K and V, of attention over it and of cross attention, in float64.

Test infrastructure only, written from the definitions in ``include/litevggt.h``: no blocking, no fusion, a loop over the
sequences, positions and heads.  Shares no code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

FP8_MAX = 448.0
EPS = 1e-6


def round_bf16(x):
    """float64 -> nearest bf16 value (ties to even), by way of the bits of float32 rounded to odd."""
    x = np.asarray(x, np.float64)
    f = x.astype(np.float32)
    up = np.abs(f.astype(np.float64)) > np.abs(x)
    f = np.where(up, np.nextafter(f, np.float32(0)), f)                # towards zero
    bits = f.view(np.uint32)
    bits = np.where(f.astype(np.float64) != x, bits | 1, bits)         # sticky
    odd = (bits >> 16) & 1
    out = ((bits + 0x7FFF + odd) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(np.isfinite(x), out, x)


def e4m3_values():
    """The 256 values of OCP E4M3 ("fn")."""
    out = []
    for code in range(256):
        s, e, m = -1.0 if code & 128 else 1.0, code >> 3 & 15, code & 7
        out.append(math.nan if e == 15 and m == 7 else s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)))
    return np.array(out)


def round_e4m3(x):
    """Nearest E4M3 value (ties to the even code), saturating; NaN stays."""
    grid = e4m3_values()[:127]                        # 0 .. 448, ascending, index = code
    a = np.minimum(np.abs(x), FP8_MAX)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), np.nan, np.copysign(grid[pick], x))


def row_exponent(row):
    """The smallest e >= -126 with max |finite x| <= 448 * 2^e; 0 for a row without a finite value over 0."""
    finite = np.abs(row[np.isfinite(row)])
    top = finite.max() if finite.size else 0.0
    if top == 0.0:
        return 0
    e = math.frexp(top)[1] - 12
    while top > FP8_MAX * 2.0 ** e:
        e += 1
    return max(e, -126)


def normed(x):
    """RMS normalisation over the last axis, rounded to bf16."""
    return round_bf16(x / np.sqrt(np.mean(x * x, -1, keepdims=True) + EPS))


class Cache:
    """Values (float64) and exponents of a pool [n_pages, kv_heads, page_tokens, head_dim]."""

    def __init__(self, n_pages, kv_heads, page_tokens, head_dim, table, e4m3):
        shape = (n_pages, kv_heads, page_tokens)
        self.k, self.v = np.zeros(shape + (head_dim,)), np.zeros(shape + (head_dim,))
        self.ke, self.ve = np.zeros(shape, np.int64), np.zeros(shape, np.int64)
        self.table, self.page, self.e4m3 = np.asarray(table), page_tokens, e4m3

    def place(self, s, pos):
        """(page, row in it) of a position, or None."""
        if pos < 0 or pos // self.page >= self.table.shape[1]:
            return None
        page = int(self.table[s, pos // self.page])
        return (page, pos % self.page) if 0 <= page < self.k.shape[0] else None

    def write(self, k, v, new_off, pos, qk_norm=False):
        for s in range(len(new_off) - 1):
            for i in range(new_off[s], new_off[s + 1]):
                at = self.place(s, pos[s] + i - new_off[s])
                if at is None:
                    continue
                page, row = at
                for pool, exps, x in ((self.k, self.ke, normed(k[i]) if qk_norm else k[i]), (self.v, self.ve, v[i])):
                    for h in range(x.shape[0]):
                        if self.e4m3:
                            e = row_exponent(x[h])
                            exps[page, h, row] = e
                            pool[page, h, row] = round_e4m3(x[h] * 2.0 ** -e) * 2.0 ** e
                        else:
                            pool[page, h, row] = x[h]

    def rows(self, s, first, count):
        """K and V of positions first .. first + count - 1 (zeros where not held), and which are held."""
        k, v = (np.zeros((count,) + self.k.shape[1:2] + self.k.shape[3:]) for _ in range(2))
        held = np.zeros(count, bool)
        for i in range(count):
            at = self.place(s, first + i)
            if at is not None:
                held[i] = True
                k[i], v[i] = self.k[at[0], :, at[1]], self.v[at[0], :, at[1]]
        return k, v, held


def attend(q, k, v, seen, scale):
    """q [n, heads, d], k, v [m, kv_heads, d], seen [n, m] -> [n, heads, d]; what a row does not see has no part in it."""
    n, heads, d = q.shape
    out = np.zeros((n, heads, d))
    if n == 0 or k.shape[0] == 0:
        return out
    group = heads // k.shape[1]
    some = seen.any(1)
    with np.errstate(all="ignore"):
        for h in range(heads):
            z = np.where(seen, q[:, h] @ k[:, h // group].T * scale, -np.inf)
            w = np.where(seen, np.exp(z - np.where(some, z.max(1), 0.0)[:, None]), 0.0)
            total = np.where(some, w.sum(1), 1.0)
            vh = v[:, h // group]
            out[:, h] = w @ np.where(np.isfinite(vh), vh, 0.0) / total[:, None]
            for t, c in np.argwhere(~np.isfinite(vh)):
                rows = seen[:, t] & (w[:, t] > 0)
                out[rows, h, c] += vh[t, c]
    return out


def cached_attention(cache, q, new_off, kv_len, frame_tokens, qk_norm=False, scale=None):
    """Rows of no sequence come back as NaN."""
    n, heads, d = q.shape
    out = np.full(q.shape, np.nan)
    q = normed(q) if qk_norm else q
    for s in range(len(new_off) - 1):
        a, b = new_off[s], new_off[s + 1]
        m = max(0, min(kv_len[s], cache.table.shape[1] * cache.page))
        k, v, held = cache.rows(s, 0, m)
        seen = np.zeros((b - a, m), bool)
        for i in range(b - a):
            p = kv_len[s] - (b - a) + i
            limit = m if frame_tokens == 0 else 0 if p < 0 else (p // frame_tokens + 1) * frame_tokens
            seen[i] = held & (np.arange(m) < limit)
        out[a:b] = attend(q[a:b], k, v, seen, scale or 1.0 / math.sqrt(d))
    return out


def cross_attention(q, q_off, k, v, kv_begin, kv_end, qk_norm=False, scale=None):
    d = q.shape[-1]
    out = np.full(q.shape, np.nan)
    if qk_norm:
        q, k = normed(q), normed(k)
    for s in range(len(q_off) - 1):
        a, b, lo, hi = q_off[s], q_off[s + 1], kv_begin[s], max(kv_begin[s], kv_end[s])
        out[a:b] = attend(q[a:b], k[lo:hi], v[lo:hi], np.ones((b - a, hi - lo), bool), scale or 1.0 / math.sqrt(d))
    return out
