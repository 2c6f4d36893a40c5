"""A cache with random rows at shuffled pages on both sides, for the tests of the E2M1 cache and of the weight that positions draw."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache_oracle as O
from oracle import stream_oracle as S
from paper_2512_04939_amd import binding as B

DTYPES = {"bf16": B.CACHE_BF16, "e4m3": B.CACHE_E4M3, "e2m1": B.CACHE_E2M1}


def rows(rng, *shape, gain=1.0):
    return O.round_bf16(rng.standard_normal(shape) * gain)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def host(t):
    return t.double().cpu().numpy()


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def packed(codes):
    """[.., d] codes -> [.., d / 2] bytes."""
    return (codes[..., ::2] | codes[..., 1::2] << 4).astype(np.uint8)


class Pool:
    def __init__(self, seed, lens, *, dtype="e2m1", heads=4, kv_heads=4, head_dim=64, page=16, frame=0, qk_norm=0, scale=0.0, holes=(), spare=3,
                 gain=1.0, more_columns=0):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.scale, self.dtype = list(lens), scale, dtype
        pages = [-(-max(n, 0) // page) for n in lens]
        self.max_pages = max(pages + [1]) + more_columns
        self.n_pages = sum(pages) + spare
        ids = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        at = 0
        for s, c in enumerate(pages):
            self.table[s, :c] = ids[at:at + c]
            at += c
        for s, c in holes:
            self.table[s, c] = -1
        self.p = B.make_cache_params(len(lens), heads, head_dim, kv_heads=kv_heads, cache_dtype=DTYPES[dtype], page_tokens=page,
                                     n_pages=self.n_pages, max_pages=self.max_pages, frame_tokens=frame, qk_norm=qk_norm, softmax_scale=scale)
        shape = (self.n_pages, kv_heads, page)
        self.o = S.Cache4(self.n_pages, kv_heads, page, head_dim, self.table) if dtype == "e2m1" else O.Cache(
            self.n_pages, kv_heads, page, head_dim, self.table, dtype == "e4m3")
        for name in ("k", "v"):
            x = rows(rng, *shape, head_dim, gain=gain)
            if dtype == "e2m1":       # random codes at random scales, quicker than rounding
                code = rng.integers(0, 16, x.shape).astype(np.uint8)
                e = rng.integers(-4, 1, shape + (head_dim // 32,))
                value = np.array([S.e2m1_value(c) for c in range(16)])
                x = value[code] * 2.0 ** np.repeat(e, 32, -1) * gain
                setattr(self.o, name + "c", code)
                setattr(self.o, name + "e", e + int(np.log2(gain)))
            elif dtype == "e4m3":
                e = rng.integers(-3, 3, shape)
                x = O.round_e4m3(x * 100) * 2.0 ** (e[..., None] - 6)
                setattr(self.o, name + "e", e - 6)
            setattr(self.o, name, x)
        self.d = self.device()

    def device(self):
        out, scales = [], []
        for name in ("k", "v"):
            x = getattr(self.o, name)
            if self.dtype == "bf16":
                out.append(dev(x))
                scales.append(None)
                continue
            e = getattr(self.o, name + "e")
            scales.append(torch.from_numpy((e + 127).astype(np.uint8)).cuda())
            if self.dtype == "e2m1":
                out.append(torch.from_numpy(packed(getattr(self.o, name + "c"))).cuda())
            else:
                out.append(torch.from_numpy(x * 2.0 ** -e[..., None]).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda())
        return B.CacheBuffers(*out, *scales, torch.from_numpy(self.table).cuda())

    def softmax_scale(self):
        return self.scale if self.scale > 0 else self.p.head_dim ** -0.5

    def score_error(self, q):
        """How far a score may be off: d products in 32 bits, each sum off by 2^-24 of sum |q k| <= |q| |k|; with the normalisation one of q's
        values may fall to the other side of a border between two bf16 values, 2^-7 of itself."""
        k = self.o.k[np.isfinite(self.o.k).all(-1)]
        qs = O.normed(q) if self.p.qk_norm else q
        qn, kn = np.sqrt((qs ** 2).sum(-1)).max(initial=0), np.sqrt((k ** 2).sum(-1)).max(initial=0)
        one = np.abs(qs).max(initial=0) * np.abs(k).max(initial=0) * 2.0 ** -7 * 2 if self.p.qk_norm else 0.0
        return self.softmax_scale() * (self.p.head_dim * 2.0 ** -24 * qn * kn + one)

    # ---- attention
    def attend(self, new, q=None, kv_len=None, tail=0):
        p, kv_len = self.p, self.lens if kv_len is None else kv_len
        off = np.concatenate([[0], np.cumsum(new)])
        n = int(off[-1]) + tail
        q = rows(self.rng, n, p.heads, p.head_dim) if q is None else q
        o = torch.full((n, p.heads, p.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n)).fill_(255)
        B.litevggt_cached_attn(p, self.d, dev(q), i32(off), i32(kv_len), o, ws)
        args = (q, off.tolist(), list(kv_len), p.frame_tokens, bool(p.qk_norm), self.softmax_scale())
        exact = O.cached_attention(self.o, *args)
        v, self.o.v = self.o.v, np.abs(self.o.v)
        spread = O.cached_attention(self.o, *args)
        self.o.v = v
        got = host(o)
        assert np.all(got[n - tail:] == 7.0)
        got, exact, spread = got[:n - tail], exact[:n - tail], spread[:n - tail]
        # a weight and the result are rounded to bf16 (2^-8 each); a score's error is a weight's, and doubled for the exponential's own
        tol = 2.0 ** -8 * np.abs(exact) + (2.0 ** -8 + 4 * self.score_error(q)) * spread + 1e-30
        assert np.array_equal(np.isfinite(got), np.isfinite(exact))
        fine = np.isfinite(exact)
        bad = (np.abs(got - exact) > tol) & fine
        assert not bad.any(), (np.argwhere(bad)[:5], np.max((np.abs(got - exact) / tol)[fine]))
        return got

    # ---- drawn weight
    def draw(self, new, q=None, kv_len=None, had="random", tail=0, in_place=False, cache=None):
        p, kv_len = self.p, self.lens if kv_len is None else kv_len
        off = np.concatenate([[0], np.cumsum(new)])
        n = int(off[-1]) + tail
        q = rows(self.rng, n, p.heads, p.head_dim) if q is None else q
        shape = (p.n_seq, p.kv_heads, p.max_pages * p.page_tokens)
        mass_in = None if had is None else self.rng.random(shape).astype(np.float32) * 1e-2
        out = np.full(shape, 5.0, np.float32)
        if in_place:
            out = mass_in
        d_in = None if mass_in is None else torch.from_numpy(mass_in.copy()).cuda()
        d_out = d_in if in_place else torch.from_numpy(out.copy()).cuda()
        ws = B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, n)).fill_(255)
        B.litevggt_cached_mass(p, cache or self.d, dev(q), i32(off), i32(kv_len), d_in, d_out, ws)
        exact = S.mass(self.o, q, off.tolist(), list(kv_len), p.frame_tokens, None if mass_in is None else mass_in.astype(np.float64),
                       out.astype(np.float64), bool(p.qk_norm), self.softmax_scale())
        got = host(d_out)
        drawn = np.abs(exact - (0.0 if mass_in is None else mass_in))
        # each weight by its score's error and its row's (at most as much), by exp2 (4 of 2^-24), its argument (the reference and c times the
        # score, below 2^6 here: 2^-18), the divisor (a sum of m, 2^-24 each at most) and the sum over rows
        rows_of = max(new, default=0) * p.heads // p.kv_heads
        rel = 2 * self.score_error(q) + 2.0 ** -17 + (max(max(kv_len), 1) + rows_of + 16) * 2.0 ** -24
        tol = rel * drawn + 2.0 ** -23 * np.abs(exact) + 1e-30
        fine = np.isfinite(exact)
        assert np.array_equal(np.isfinite(got), fine)
        bad = (np.abs(got - exact) > tol) & fine
        assert not bad.any(), (np.argwhere(bad)[:5], np.max((np.abs(got - exact) / tol)[fine]))
        return got
