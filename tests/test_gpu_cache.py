"""The paged cache, attention over it and cross attention on the GPU against the plain implementation in 64 bits.

Tolerances.  A weight is rounded to bf16 for the second product (off by at most 2^-8 of itself), as is the result (2^-8),
so an output is off by at most 2^-8 (|o| + sum w |v| / sum w); scores are sums of d products in fp32, off by d 2^-24 of
sum |q k| at most, which the exponential turns into that share of a weight (times the scale).  `bound` is that, doubled in
its last term for the exponential's own error.  With qk_norm a normalised value on the border of two bf16 values
may fall to the other side in 32 bits: one of a row's d products then moves by 2^-7 of itself, counted for q and k."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2512_04939_amd import binding as B

pytestmark = pytest.mark.gpu


def rows(rng, *shape, gain=1.0):
    return O.round_bf16(rng.standard_normal(shape) * gain)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).cuda()


def host(t):
    return t.double().cpu().numpy()


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def bound(oracle, v_abs_out, out, q, k, scale, qk_norm):
    d = q.shape[-1]
    qm, km = np.nanmax(np.abs(q), initial=0), np.max(np.abs(k[np.isfinite(k)]), initial=0)
    score = scale * d * 2.0 ** -24 * d * qm * km * 2
    if qk_norm:
        score += scale * 2 * 2.0 ** -7 * qm * km
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * score) * v_abs_out + 1e-30


class Case:
    """A cache with random rows at shuffled pages, on both sides."""

    def __init__(self, seed, lens, *, heads=4, kv_heads=4, head_dim=64, e4m3=False, page=16, frame=0, qk_norm=0, scale=0.0,
                 holes=(), spare=3, gain=1.0):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.scale = list(lens), scale
        pages = [-(-max(n, 0) // page) for n in lens]
        self.max_pages = max(pages + [1])
        self.n_pages = sum(pages) + spare
        ids = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        at = 0
        for s, c in enumerate(pages):
            self.table[s, :c] = ids[at:at + c]
            at += c
        for s, c in holes:
            self.table[s, c] = -1
        self.p = B.make_cache_params(len(lens), heads, head_dim, kv_heads=kv_heads, cache_dtype=B.CACHE_E4M3 if e4m3 else B.CACHE_BF16,
                                     page_tokens=page, n_pages=self.n_pages, max_pages=self.max_pages, frame_tokens=frame,
                                     qk_norm=qk_norm, softmax_scale=scale)
        self.o = O.Cache(self.n_pages, kv_heads, page, head_dim, self.table, e4m3)
        shape = (self.n_pages, kv_heads, page)
        for name in ("k", "v"):
            x = rows(rng, *shape, head_dim, gain=gain)
            if e4m3:
                e = rng.integers(-3, 3, shape)
                x = O.round_e4m3(x * 100) * 2.0 ** (e[..., None] - 6)
                setattr(self.o, name + "e", e - 6)
            setattr(self.o, name, x)
        self.d = self.device()

    def device(self):
        out = []
        for name in ("k", "v"):
            x = getattr(self.o, name)
            if self.o.e4m3:
                x = x * 2.0 ** -getattr(self.o, name + "e")[..., None]
                out.append(torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).cuda())
            else:
                out.append(dev(x))
        scales = [torch.from_numpy((getattr(self.o, n) + 127).astype(np.uint8)).cuda() if self.o.e4m3 else None for n in ("ke", "ve")]
        return B.CacheBuffers(*out, *scales, torch.from_numpy(self.table).cuda())

    def attend(self, new, q=None, kv_len=None, ws=None, tail=0):
        """(device output, exact output, bound) for `new` tokens per sequence; `tail` rows of no sequence behind them."""
        p, kv_len = self.p, self.lens if kv_len is None else kv_len
        off = np.concatenate([[0], np.cumsum(new)])
        n = int(off[-1]) + tail
        if q is None:
            q = rows(self.rng, n, p.heads, p.head_dim)
        o = torch.full((n, p.heads, p.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n)) if ws is None else ws
        ws.fill_(255)
        B.litevggt_cached_attn(p, self.d, dev(q), i32(off), i32(kv_len), o, ws)
        scale = self.scale if self.scale > 0 else p.head_dim ** -0.5
        args = (q, off.tolist(), list(kv_len), p.frame_tokens, bool(p.qk_norm), scale)
        exact = O.cached_attention(self.o, *args)
        v, self.o.v = self.o.v, np.abs(self.o.v)
        spread = O.cached_attention(self.o, *args)
        self.o.v = v
        qs = O.normed(q) if p.qk_norm else q
        got = host(o)
        if tail:
            assert np.all(got[n - tail:] == 7.0)
            got, exact, spread = got[:n - tail], exact[:n - tail], spread[:n - tail]
        return got, exact, bound(self.o, spread, exact, qs, self.o.k, scale, p.qk_norm)

    def check(self, new, **kw):
        got, exact, tol = self.attend(new, **kw)
        assert got.shape == exact.shape
        assert np.array_equal(np.isfinite(got), np.isfinite(exact))
        bad = np.abs(got - exact) > tol
        assert not bad[np.isfinite(exact)].any(), (np.argwhere(bad)[:5], np.nanmax(np.abs(got - exact) / tol))
        return got


# ------------------------------------------------------------------ the cache
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim,heads,page,new,pos", [
    (64, 1, 16, [1], [0]), (64, 16, 64, [1], [500]), (64, 5, 16, [3, 0, 21, 1], [15, 7, 0, 40]), (128, 2, 32, [70, 5], [31, 0]),
    (64, 3, 1024, [700], [900]), (128, 4, 16, [2] * 70, list(range(70))),
])
def test_write(e4m3, dim, heads, page, new, pos):
    c = Case(1, [p + n for p, n in zip(pos, new)], heads=heads, kv_heads=heads, head_dim=dim, e4m3=e4m3, page=page)
    rng = np.random.default_rng(2)
    n = sum(new)
    off = [0] + np.cumsum(new).tolist()
    k, v = rows(rng, n + 2, heads, dim), rows(rng, n + 2, heads, dim, gain=30.0)
    if n > 2:
        k[1] = 0.0
        v[0, 0, :4] = [2.0 ** -130, -2.0 ** 100, 0.0, 2.0 ** -126]
    # rows of no sequence behind the last; K and V as slices of one projection
    both = dev(np.concatenate([k.reshape(n + 2, -1), v.reshape(n + 2, -1)], 1))
    kd, vd = both[:, :heads * dim].unflatten(1, (heads, dim)), both[:, heads * dim:].unflatten(1, (heads, dim))
    B.litevggt_cache_write(c.p, c.d, kd, vd, i32(off), i32(pos))
    c.o.write(k, v, off, pos)
    want = c.device()
    for name in ("k", "v") + (("k_scale", "v_scale") if e4m3 else ()):
        assert torch.equal(getattr(c.d, name).view(torch.uint8), getattr(want, name).view(torch.uint8)), name


@pytest.mark.parametrize("dim", [64, 128])
def test_write_e4m3_of_values_that_are_not_finite(dim):
    c = Case(3, [16], heads=1, kv_heads=1, head_dim=dim, e4m3=True)
    x = np.ones((16, 1, dim))
    x[0, 0, 3], x[1, 0, 5], x[2, 0, 0] = np.inf, -np.inf, np.nan
    x[3] = np.inf
    x[4] = np.nan
    x[5] = 3.3895e38                              # the largest bf16 value, about
    x[6] = 2.0 ** -133
    x[7, 0, 0] = 450.0
    x = O.round_bf16(x)
    B.litevggt_cache_write(c.p, c.d, dev(x), dev(x), i32([0, 16]), i32([0]))
    c.o.write(x, x, [0, 16], [0])
    got = c.d.v[c.table[0, 0], 0].view(torch.float8_e4m3fn).double().cpu().numpy()
    e = c.d.v_scale[c.table[0, 0], 0].cpu().numpy().astype(int) - 127
    assert e.tolist() == c.o.ve[c.table[0, 0], 0].tolist()
    assert np.array_equal(got * 2.0 ** e[:, None], c.o.v[c.table[0, 0], 0], equal_nan=True)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_write_normalised_k(e4m3, dim):
    c = Case(4, [50], heads=3, kv_heads=3, head_dim=dim, e4m3=e4m3, qk_norm=1)
    x = rows(np.random.default_rng(5), 50, 3, dim, gain=9.0)
    B.litevggt_cache_write(c.p, c.d, dev(x), dev(x), i32([0, 50]), i32([0]))
    c.o.write(x, x, [0, 50], [0], qk_norm=True)
    k = host(c.d.k.view(torch.float8_e4m3fn) if e4m3 else c.d.k)
    if e4m3:
        k = k * 2.0 ** (c.d.k_scale.cpu().numpy().astype(float) - 127)[..., None]
    # a bf16 value on the border of two may fall to the other side, and move to the next code
    off = np.abs(k - c.o.k)
    assert np.all(off <= (2.0 ** -3 if e4m3 else 2.0 ** -7) * np.abs(c.o.k)) and np.mean(off > 0) < 1e-2


def test_write_leaves_out_what_has_no_page():
    """Holes, a page number beyond the pool, positions before 0 and beyond the table."""
    c = Case(6, [64, 64], heads=2, kv_heads=2, holes=[(0, 1)])
    c.table[1, 2] = c.o.table[1, 2] = c.n_pages
    c.d = c.device()
    k = rows(np.random.default_rng(7), 100, 2, 64)
    off, pos = [0, 60, 100], [-5, 30]
    B.litevggt_cache_write(c.p, c.d, dev(k), dev(k), i32(off), i32(pos))
    c.o.write(k, k, off, pos)
    assert np.array_equal(host(c.d.k), c.o.k) and np.array_equal(host(c.d.v), c.o.v)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim,heads,page,first,count", [
    (64, 4, 16, [0, 3, 9], [40, 0, 13]), (128, 1, 32, [5], [1]), (64, 16, 128, [100, 0], [200, 7]), (128, 3, 16, [0] * 66, [1, 4] * 33),
])
def test_read(e4m3, dim, heads, page, first, count):
    lens = [f + n for f, n in zip(first, count)]
    c = Case(8, lens, heads=heads, kv_heads=heads, head_dim=dim, e4m3=e4m3, page=page, holes=[(0, 0)])
    off = [0] + np.cumsum(count).tolist()
    n = off[-1] + 3
    k = torch.full((n, heads, dim), 5.0, dtype=torch.bfloat16, device="cuda")
    wide = torch.full((n, heads * dim + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    B.litevggt_cache_read(c.p, c.d, i32(first), i32(off), k, wide[:, :heads * dim])
    k, v = host(k), host(wide)
    assert np.all(k[n - 3:] == 5.0) and np.all(v[n - 3:] == 5.0) and np.all(v[:, heads * dim:] == 5.0)
    for s, (f, m) in enumerate(zip(first, count)):
        rk, rv, _ = c.o.rows(s, f, m)
        assert np.array_equal(k[off[s]:off[s + 1]], rk)
        assert np.array_equal(v[off[s]:off[s + 1], :heads * dim].reshape(m, heads, dim), rv)


def test_pools_over_four_gigabytes():
    """Row offsets pass 2^32 bytes and 2^31 elements."""
    n_pages, heads, page, dim = 5000, 16, 256, 128              # 5.2 GB of bf16 for K, as much for V
    p = B.make_cache_params(1, heads, dim, page_tokens=page, n_pages=n_pages, max_pages=4)
    pool = [torch.empty(n_pages, heads, page, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = [n_pages - 1, 7, n_pages - 2, 4099]
    d = B.CacheBuffers(*pool, None, None, torch.tensor([table], dtype=torch.int32, device="cuda"))
    rng = np.random.default_rng(9)
    k, v, q = (rows(rng, 1000, heads, dim) for _ in range(3))
    B.litevggt_cache_write(p, d, dev(k), dev(v), i32([0, 1000]), i32([0]))
    assert np.array_equal(host(pool[0][table[0]]), k[:256].transpose(1, 0, 2))
    out = [torch.zeros(1000, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.litevggt_cache_read(p, d, i32([0]), i32([0, 1000]), *out)
    assert np.array_equal(host(out[0]), k) and np.array_equal(host(out[1]), v)
    for n in (3, 150):
        o = torch.zeros(n, heads, dim, dtype=torch.bfloat16, device="cuda")
        B.litevggt_cached_attn(p, d, dev(q[:n]), i32([0, n]), i32([1000]), o, B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n)))
        args = (np.ones((n, 1000), bool), dim ** -0.5)
        exact, spread = O.attend(q[:n], k, v, *args), O.attend(q[:n], k, np.abs(v), *args)
        assert np.all(np.abs(host(o) - exact) <= bound(None, spread, exact, q[:n], k, dim ** -0.5, False))


# ------------------------------------------------------------------ attention over the cache
CACHED = [
    # lens, new, heads, kv_heads, frame
    ([1], [1], 1, 1, 0), ([1], [1], 4, 2, 1), ([17], [1], 2, 2, 1), ([394], [1], 4, 4, 1), ([1000], [5], 16, 16, 0),
    ([33, 0, 500, 64], [1, 0, 1, 1], 8, 2, 1), ([700, 31], [3, 31], 6, 2, 1), ([300], [300], 2, 1, 1), ([522], [261], 2, 2, 261),
    ([2100, 130], [1, 2], 3, 1, 0), ([129], [128], 2, 2, 0), ([260, 777], [200, 400], 2, 2, 50), ([600], [600], 1, 1, 7),
    ([200] * 70, [1, 2] * 35, 2, 1, 1), ([1500], [40], 12, 4, 64), ([513], [513], 4, 4, 0),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,new,heads,kv,frame", CACHED)
def test_cached_attention(lens, new, heads, kv, frame, dim, e4m3):
    page = (16, 32, 64, 128)[len(lens) % 2 + 2 * (heads % 2)]
    Case(10, lens, heads=heads, kv_heads=kv, head_dim=dim, e4m3=e4m3, page=page, frame=frame).check(new, tail=1)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_cached_attention_long_axis_cut_among_workgroups(new, dim, e4m3):
    Case(11, [9000, 5, 3333], heads=2, kv_heads=1, head_dim=dim, e4m3=e4m3, page=16, frame=1).check([new, 1, new])


@pytest.mark.parametrize("new", [1, 33, 200])
def test_cached_attention_one_key_axis_in_many_pieces(new):
    Case(12, [40000], heads=1, kv_heads=1, page=1024, frame=0).check([new])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [2, 100])
def test_cached_attention_normalised_q_and_scale(new, e4m3):
    Case(13, [600], heads=4, kv_heads=2, e4m3=e4m3, qk_norm=1, scale=0.31, gain=1.0).check([new])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new,frame", [(1, 0), (20, 16), (200, 16), (200, 1)])
def test_pages_that_are_not_held(new, frame, e4m3):
    """Every page from the third to the eighth, the last one and one in the middle; a sequence without any: zeros."""
    holes = [(0, c) for c in (2, 3, 4, 5, 6, 7, 20, 37)] + [(1, c) for c in range(20)]
    got = Case(14, [600, 310], heads=2, kv_heads=2, page=16, frame=frame, e4m3=e4m3, holes=holes).check([new, new])
    assert np.all(got[new:] == 0)


def test_more_queries_than_positions_and_lengths_out_of_range():
    """Queries before position 0 see nothing; a length beyond the table is cut to it; a negative one is none."""
    c = Case(15, [160, 160, 160], heads=2, kv_heads=1, page=16, frame=1)
    got = c.check([200, 3, 4], kv_len=[160, 5000, -7])
    assert np.all(got[:40] == 0) and np.all(got[203:] == 0)
    Case(15, [160], heads=2, kv_heads=1, page=16, frame=0).check([200], kv_len=[160])


@pytest.mark.parametrize("new", [1, 8, 300])
@pytest.mark.parametrize("dim", [64, 128])
def test_references_raised_many_times(new, dim):
    """Scores that climb by hundreds of binades along the key axis, then fall; queries of both signs and of no size."""
    c = Case(16, [800], heads=2, kv_heads=1, head_dim=dim, page=16)
    ramp = np.concatenate([np.linspace(0, 8, 500), np.linspace(8, -8, 300)])
    for t in range(800):
        page, row = c.o.place(0, t)
        c.o.k[page, 0, row] = O.round_bf16(ramp[t] * np.ones(dim) + 0.01 * c.rng.standard_normal(dim))
    c.d = c.device()
    q = O.round_bf16(np.where(np.arange(new) % 3 == 0, 10.0, np.where(np.arange(new) % 3 == 1, -10.0, 0.0))[:, None, None]
                     * np.ones((new, 2, dim)))
    got, exact, tol = c.attend([new], q=q)
    # scores up to 8 * 10 * dim * scale = 640 (64) or 905 (128): q k is exact to d 2^-24 relative, 2^-18 * 900 = 0.0035 on a score,
    # which the bound (of the largest |q k|) already counts
    assert np.all(np.abs(got - exact) <= tol)


@pytest.mark.parametrize("new", [3, 100, 300])
def test_values_that_are_not_finite_stay_with_those_who_see_them(new):
    """Infinities and NaN in K and V behind the end, in pages not held and in tokens that a query does not see."""
    c = Case(17, [320, 300], heads=2, kv_heads=2, page=16, frame=1, holes=[(0, 2)])
    wild = [np.inf, -np.inf, np.nan]
    for i, t in enumerate([318, 319, 300, 301]):
        page, row = c.o.place(0, t)
        c.o.v[page, 0, row, 5 * i] = wild[i % 3]
    page, row = c.o.place(1, 298)
    c.o.k[page, 1, row, 3] = np.nan
    page, row = c.o.place(1, 299)
    c.o.v[page, :, row] = np.nan
    page = c.o.place(1, 299)[0]
    c.o.k[page, :, 300 % 16:] = np.nan           # behind the end
    c.o.v[page, :, 300 % 16:] = np.inf
    hole = [p for p in range(c.n_pages) if p not in c.table][0]
    c.o.k[hole], c.o.v[hole] = np.nan, np.inf
    c.d = c.device()
    got, exact, tol = c.attend([new, new])
    ok = np.isfinite(exact)
    assert np.array_equal(ok, np.isfinite(got))
    assert np.all(np.abs(got - exact)[ok] <= np.nan_to_num(tol, nan=np.inf)[ok])
    assert np.isfinite(got[:new - 20]).all() if new > 20 else True


def test_two_calls_give_the_same_bits_whatever_the_workspace_holds():
    c = Case(18, [5000, 700], heads=4, kv_heads=2, page=64, frame=1)
    q = rows(c.rng, 12, 4, 64)
    a, _, _ = c.attend([6, 6], q=q)
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, 12) + 4096)
    b, _, _ = c.attend([6, 6], q=q, ws=ws)
    assert np.array_equal(a, b)


# ------------------------------------------------------------------ cross attention
CROSS = [
    # queries, (begin, end) of the states, states, heads, kv_heads
    ([1], [(0, 1)], 1, 1, 1), ([5], [(0, 0)], 3, 2, 1), ([5, 5], [(0, 1374), (1374, 2748)], 2748, 4, 4),
    ([3, 0, 200, 1], [(0, 700), (5, 9), (9, 9), (100, 163)], 700, 8, 2), ([130], [(1, 66)], 70, 2, 2), ([700], [(0, 900)], 900, 2, 1),
    ([40] * 3, [(0, 500)] * 3, 500, 6, 2), ([1] * 80, [(i, 3 * i) for i in range(80)], 240, 2, 2), ([260], [(0, 6000)], 6000, 1, 1),
]


def run_cross(rng, nq, ranges, m, heads, kv, dim, qk_norm=0, scale=0.0, fused=False, q=None, k=None, v=None):
    off = [0] + np.cumsum(nq).tolist()
    n = off[-1] + 2                       # two rows of no sequence
    q = rows(rng, n, heads, dim) if q is None else q
    k = rows(rng, m, kv, dim) if k is None else k
    v = rows(rng, m, kv, dim) if v is None else v
    if fused:
        both = dev(np.concatenate([k.reshape(m, -1), v.reshape(m, -1)], 1))
        kd, vd = both[:, :kv * dim], both[:, kv * dim:]
    else:
        kd, vd = dev(k), dev(v)
    p = B.make_cross_params(len(nq), heads, dim, kv_heads=kv, qk_norm=qk_norm, softmax_scale=scale)
    o = torch.full((n, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, n, m)).fill_(255)
    begin, end = [r[0] for r in ranges], [r[1] for r in ranges]
    B.litevggt_cross_attn(p, dev(q), i32(off), kd, vd, i32(begin), i32(end), o, ws)
    got = host(o)
    assert np.all(got[-2:] == 7.0)
    s = scale or dim ** -0.5
    lo, hi = np.clip(begin, 0, m), np.clip(end, 0, m)
    exact = O.cross_attention(q, off, k, v, lo, hi, bool(qk_norm), s)[:-2]
    spread = O.cross_attention(q, off, k, np.abs(v), lo, hi, bool(qk_norm), s)[:-2]
    tol = bound(None, spread, exact, O.normed(q) if qk_norm else q, O.normed(k) if qk_norm else k, s, qk_norm)
    return got[:-2], exact, tol


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,ranges,m,heads,kv", CROSS)
def test_cross_attention(nq, ranges, m, heads, kv, dim, fused):
    got, exact, tol = run_cross(np.random.default_rng(20), nq, ranges, m, heads, kv, dim, fused=fused)
    assert np.all(np.abs(got - exact) <= tol), np.max(np.abs(got - exact) / tol)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq", [4, 150])
def test_cross_attention_normalised(nq, dim):
    got, exact, tol = run_cross(np.random.default_rng(21), [nq], [(3, 400)], 401, 4, 2, dim, qk_norm=1, scale=0.2, fused=True)
    assert np.all(np.abs(got - exact) <= tol), np.max(np.abs(got - exact) / tol)


def test_cross_attention_ranges_beyond_the_states_and_no_states():
    got, exact, tol = run_cross(np.random.default_rng(22), [3, 3], [(-4, 20), (10, 99)], 25, 2, 2, 64)
    assert np.all(np.abs(got - exact) <= tol)
    p = B.make_cross_params(1, 2, 64)
    o = torch.full((4, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.ones_like(o)
    B.litevggt_cross_attn(p, q, i32([0, 4]), None, None, i32([0]), i32([0]), o, B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, 4, 0)))
    assert torch.all(o == 0)


def test_cross_attention_states_around_a_range_have_no_part():
    rng = np.random.default_rng(23)
    k, v = rows(rng, 300, 2, 64), rows(rng, 300, 2, 64)
    k[:37] = k[230:] = np.nan
    v[:37] = v[230:] = np.inf
    for n in (2, 200):
        got, exact, tol = run_cross(rng, [n], [(37, 230)], 300, 2, 2, 64, k=k, v=v)
        assert np.isfinite(got).all() and np.all(np.abs(got - exact) <= tol)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("e4m3", [False, True])
def test_frames_as_they_arrive(e4m3):
    """Four frames of 261 tokens: each is written and attends to what is there; then five queries attend to the cache read back as states,
    and single tokens to the cache itself.  The frames' outputs are those of one call over the whole sequence."""
    T, F, heads, dim = 261, 4, 4, 64
    n = T * F
    c = Case(30, [n], heads=heads, kv_heads=heads, page=64, frame=T, e4m3=e4m3)
    rng = np.random.default_rng(31)
    q, k, v = (rows(rng, n, heads, dim) for _ in range(3))
    qd, kd, vd = dev(q), dev(k), dev(v)
    o, whole = torch.empty_like(qd), torch.empty_like(qd)
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, n))
    for f in range(F):
        part = slice(f * T, (f + 1) * T)
        B.litevggt_cache_write(c.p, c.d, kd[part], vd[part], i32([0, T]), i32([f * T]))
        B.litevggt_cached_attn(c.p, c.d, qd[part], i32([0, T]), i32([(f + 1) * T]), o[part], ws)
    B.litevggt_cached_attn(c.p, c.d, qd, i32([0, n]), i32([n]), whole, ws)
    c.o.write(k, v, [0, n], [0])
    exact = O.cached_attention(c.o, q, [0, n], [n], T)
    ck, cv, _ = c.o.rows(0, 0, n)
    c.o.v = np.abs(c.o.v)
    tol = bound(None, O.cached_attention(c.o, q, [0, n], [n], T), exact, q, c.o.k, 0.125, False)
    for got in (host(o), host(whole)):
        assert np.all(np.abs(got - exact) <= tol)
    back = [torch.empty(n, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.litevggt_cache_read(c.p, c.d, i32([0]), i32([0, n]), *back)
    assert np.array_equal(host(back[0]), ck) and np.array_equal(host(back[1]), cv)
    xp = B.make_cross_params(1, heads, dim)
    x = torch.empty(5, heads, dim, dtype=torch.bfloat16, device="cuda")
    B.litevggt_cross_attn(xp, qd[:5], i32([0, 5]), *back, i32([0]), i32([n]), x, B.alloc_ws(B.litevggt_cross_attn_ws_bytes(xp, 5, n)))
    args = (np.ones((5, n), bool), 0.125)
    exact, spread = O.attend(q[:5], ck, cv, *args), O.attend(q[:5], ck, np.abs(cv), *args)
    assert np.all(np.abs(host(x) - exact) <= bound(None, spread, exact, q[:5], ck, 0.125, False))


def test_captured_and_replayed_with_other_lengths():
    """A write and the attention over the cache in a graph, replayed while the sequences grow, with eager calls of other
    sizes between the replays that use the same workspace."""
    c = Case(32, [400, 300], heads=4, kv_heads=2, page=16, frame=1)
    rng = np.random.default_rng(33)
    p, ws = c.p, B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, 64))
    k, v, q = (torch.zeros(2, h, 64, dtype=torch.bfloat16, device="cuda") for h in (2, 2, 4))
    off, pos, length, o = i32([0, 1, 2]), i32([0, 0]), i32([1, 1]), torch.zeros_like(q)

    def step():
        B.litevggt_cache_write(p, c.d, k, v, off, pos)
        B.litevggt_cached_attn(p, c.d, q, off, length, o, ws)

    step()                                     # position 0 of both sequences holds zeros now
    c.o.write(np.zeros((2, 2, 64)), np.zeros((2, 2, 64)), [0, 1, 2], [0, 0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for at in ([300, 200], [301, 201], [350, 0], [15, 16], [399, 299]):
        x = [rows(rng, 2, h, 64) for h in (2, 2, 4)]
        for t, y in zip((k, v, q), x):
            t.copy_(dev(y))
        pos.copy_(i32(at))
        length.copy_(i32([a + 1 for a in at]))
        graph.replay()
        got = o.clone()
        c.o.write(x[0], x[1], [0, 1, 2], at)
        exact = O.cached_attention(c.o, x[2], [0, 1, 2], [a + 1 for a in at], 1)
        v0, c.o.v = c.o.v, np.abs(c.o.v)
        tol = bound(None, O.cached_attention(c.o, x[2], [0, 1, 2], [a + 1 for a in at], 1), exact, x[2], c.o.k, 0.125, False)
        c.o.v = v0
        assert np.all(np.abs(host(got) - exact) <= tol), at
        c.attend([20, 30], ws=ws, kv_len=[60, 70])
        torch.cuda.synchronize()


def test_on_a_stream_of_its_own():
    c = Case(34, [900], heads=2, kv_heads=2, page=32, frame=0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.check([3])
        c.check([200])
