"""Plain CPU implementation of what keeps a stream's cache small, in float64: rotary positions with several axes, a cache held in E2M1,
the attention weight that positions draw, the eviction of pages.

Test infrastructure only, written from the definitions in ``include/litevggt.h``.  Shares no code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

from . import cache_oracle as O

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
BLOCK = 32


def e2m1_code(x):
    """The code (0 .. 15) of the E2M1 value next to x, of two as near the one with the even code."""
    a = abs(x)
    best = min(range(8), key=lambda c: (abs(a - E2M1[c]), c % 2))
    return best | (8 if math.copysign(1.0, x) < 0 else 0)


def e2m1_value(code):
    return math.copysign(E2M1[code & 7], -1.0 if code & 8 else 1.0)


def block_exponent(block):
    """The smallest e >= -126 with max |finite x| <= 6 * 2^e; 0 for a block without a finite value over 0; None if there is a NaN."""
    if np.isnan(block).any():
        return None
    finite = np.abs(block[np.isfinite(block)])
    top = finite.max() if finite.size else 0.0
    if top == 0.0:
        return 0
    e = math.frexp(top)[1] - 5
    while top > 6.0 * 2.0 ** e:
        e += 1
    return max(e, -126)


def round_blocks(x):
    """Rows [..., d] -> (values that they are held as, exponents [..., d / 32], codes [..., d])."""
    flat = np.asarray(x, np.float64).reshape(-1, BLOCK)
    out, exps, codes = np.empty_like(flat), np.empty(len(flat), np.int64), np.zeros(flat.shape, np.uint8)
    for i, block in enumerate(flat):
        e = block_exponent(block)
        if e is None:
            out[i], exps[i] = np.nan, 128
            continue
        exps[i] = e
        z = np.clip(block / 2.0 ** e, -6.0, 6.0)
        codes[i] = [e2m1_code(v) for v in z]
        out[i] = [e2m1_value(c) * 2.0 ** e for c in codes[i]]
    shape = np.asarray(x).shape
    return out.reshape(shape), exps.reshape(shape[:-1] + (shape[-1] // BLOCK,)), codes.reshape(shape)


class Cache4(O.Cache):
    """A pool held in E2M1: values, codes and exponents."""

    def __init__(self, n_pages, kv_heads, page_tokens, head_dim, table):
        super().__init__(n_pages, kv_heads, page_tokens, head_dim, table, False)
        shape = (n_pages, kv_heads, page_tokens)
        self.kc, self.vc = np.zeros(shape + (head_dim,), np.uint8), np.zeros(shape + (head_dim,), np.uint8)
        self.ke, self.ve = (np.zeros(shape + (head_dim // BLOCK,), np.int64) for _ in range(2))

    def fill(self, name, x):
        value, e, code = round_blocks(x)
        setattr(self, name, value)
        setattr(self, name + "e", e)
        setattr(self, name + "c", code)

    def write(self, k, v, new_off, pos, qk_norm=False):
        for s in range(len(new_off) - 1):
            for i in range(new_off[s], new_off[s + 1]):
                at = self.place(s, pos[s] + i - new_off[s])
                if at is None:
                    continue
                page, row = at
                for name, x in (("k", O.normed(k[i]) if qk_norm else k[i]), ("v", v[i])):
                    value, e, code = round_blocks(x)
                    getattr(self, name)[page, :, row] = value
                    getattr(self, name + "e")[page, :, row] = e
                    getattr(self, name + "c")[page, :, row] = code


def mass(cache, q, new_off, kv_len, frame_tokens, mass_in, out, qk_norm=False, scale=None):
    """What `out` [n_seq, kv_heads, positions] becomes."""
    n, heads, d = q.shape
    kv = cache.k.shape[1]
    q = O.normed(q) if qk_norm else q
    scale = scale or 1.0 / math.sqrt(d)
    out = out.copy()
    for s in range(len(kv_len)):
        a, b = new_off[s], new_off[s + 1]
        m = max(0, min(kv_len[s], cache.table.shape[1] * cache.page))
        k, _, held = cache.rows(s, 0, m)
        drawn = np.zeros((kv, m))
        for i in range(a, b):
            p = kv_len[s] - b + i
            limit = m if frame_tokens == 0 else 0 if p < 0 else (p // frame_tokens + 1) * frame_tokens
            seen = held & (np.arange(m) < limit)
            if not seen.any():
                continue
            for h in range(heads):
                z = k[seen, h // (heads // kv)] @ q[i, h] * scale
                with np.errstate(all="ignore"):
                    w = np.exp(z - z.max())
                    drawn[h // (heads // kv), seen] += w / w.sum()
        had = 0.0 if mass_in is None else mass_in[s, :, :m]
        out[s, :, :m] = np.where(held, had + drawn, 0.0)
    return out


def evict(table, n_pages, page_tokens, kv_len, masses, keep, first_pages, last_pages):
    """(table, freed [n_seq, columns], count [n_seq])."""
    table, freed = np.array(table), np.full_like(table, -1)
    counts = np.zeros(len(kv_len), np.int64)
    for s, length in enumerate(kv_len):
        length = max(0, min(int(length), table.shape[1] * page_tokens))
        used = -(-length // page_tokens)
        held = [j for j in range(used) if 0 <= table[s, j] < n_pages]
        weight = {}
        for j in held:
            x = masses[s, :, j * page_tokens:min((j + 1) * page_tokens, length)].astype(np.float64)
            total = math.fsum(x.ravel()) if np.isfinite(x).all() else float(x.sum())
            weight[j] = (math.isnan(total), 0.0 if math.isnan(total) else total)
        may = sorted((j for j in held if first_pages <= j < used - last_pages), key=lambda j: (weight[j], j))
        gone = sorted(may[:max(0, len(held) - max(int(keep[s]), 0))])
        freed[s, :len(gone)] = table[s, gone]
        table[s, gone] = -1
        counts[s] = len(gone)
    return table, freed, counts


def rope(x, pos, pairs, pairing, joint, inverse, base=None, freq=None):
    """x [n, heads, d], pos [n, axes]; pairing 0: halves of an axis' channels, 1: halves of all that turn, 2: neighbours."""
    y, total, first = np.array(x, np.float64), sum(pairs), 0
    for a, p in enumerate(pairs):
        for j in range(p):
            i = first + j
            f = freq[i] if freq is not None else float(base) ** (-(i / total) if joint else -(j / p))
            c1, c2 = ((2 * first + j, 2 * first + p + j), (i, total + i), (2 * i, 2 * i + 1))[pairing]
            turns = np.array([math.fmod(int(t) * f, 2 * math.pi) for t in pos[:, a]])
            c, s = np.cos(turns)[:, None], np.sin(turns)[:, None] * (-1 if inverse else 1)
            y[..., c1], y[..., c2] = x[..., c1] * c - x[..., c2] * s, x[..., c2] * c + x[..., c1] * s
        first += p
    return y
