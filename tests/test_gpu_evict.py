"""Eviction on the GPU against the plain implementation (exact), and a stream that runs rotation, cache, attention, drawn weight and eviction
together."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from oracle import stream_oracle as S
from paper_2512_04939_amd import binding as B

from stream_cases import dev, host, i32, rows

pytestmark = pytest.mark.gpu


def run(table, n_pages, page, lens, mass, keep, first=0, last=0, in_place=False, slack=0):
    n_seq, columns = table.shape
    p = B.make_cache_params(n_seq, mass.shape[1], 64, page_tokens=page, n_pages=n_pages, max_pages=columns)
    t = torch.from_numpy(table.copy()).cuda()
    out = t if in_place else torch.full_like(t, 99)
    freed, count = torch.full_like(t, 99), torch.full((n_seq,), 99, dtype=torch.int32, device="cuda")
    ws = B.alloc_ws(B.litevggt_cache_evict_ws_bytes(p)).fill_(255)
    B.litevggt_cache_evict(p, t, i32(lens), torch.from_numpy(mass).cuda(), i32(keep), first, last, out, freed, count, ws)
    got = [x.cpu().numpy() for x in (out, freed, count)]
    want = S.evict(table, n_pages, page, lens, mass, keep, first, last)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    return got


def tables(rng, pages, columns, n_pages, holes=0.1):
    t = np.full((len(pages), columns), -1, np.int32)
    ids = rng.permutation(n_pages)
    at = 0
    for s, c in enumerate(pages):
        t[s, :c] = np.where(rng.random(c) < holes, -1, ids[at:at + c])
        at += c
    return t


@pytest.mark.parametrize("page", [16, 64, 256, 512, 1024])
@pytest.mark.parametrize("heads,pages", [(1, [1]), (3, [7, 0, 1, 40]), (16, [300, 5]), (2, [1100, 2049])])
def test_evict(page, heads, pages):
    if page > 64 and max(pages) > 300:
        pages = [x // 8 for x in pages]
    rng = np.random.default_rng(page + heads)
    columns = max(pages) + 2
    n_pages = sum(pages) + 2
    t = tables(rng, pages, columns, n_pages)
    lens = [max(0, c * page - int(rng.integers(0, page))) for c in pages]
    mass = (rng.random((len(pages), heads, columns * page)) ** 2).astype(np.float32)
    mass *= np.exp(2 * rng.standard_normal((len(pages), 1, columns))).repeat(page, 2).astype(np.float32)
    mass *= (rng.random((len(pages), 1, columns)) < 0.8).repeat(page, 2)          # pages that drew nothing: ties
    for share, first, last in ((0.5, 0, 0), (0.0, 1, 2), (0.9, 0, 1), (1.1, 0, 0), (-1, 3, 0), (0.3, 10 ** 6, 0), (0.3, 0, 10 ** 6)):
        run(t, n_pages, page, lens, mass, [int(share * c) for c in pages], first, last)
    run(t, n_pages, page, lens, mass, [c // 3 for c in pages], 1, 1, in_place=True)


def test_ties_signs_and_what_is_not_finite():
    rng = np.random.default_rng(5)
    t = tables(rng, [1500], 1500, 1500, holes=0.0)
    length = [1500 * 16]
    page = lambda v: np.repeat(v.astype(np.float32), 16)[None, None]       # noqa: E731
    for v in (np.zeros(1500), np.full(1500, 0.1), rng.integers(0, 3, 1500), rng.standard_normal(1500), np.where(rng.random(1500) < 0.5, -0.0, 0.0),
              np.where(rng.random(1500) < 0.3, np.inf, 1.0), np.where(rng.random(1500) < 0.3, np.nan, -1.0), np.full(1500, np.nan),
              np.where(rng.random(1500) < 0.3, -np.inf, rng.random(1500)), 1.0 + 2.0 ** -23 * rng.integers(0, 5, 1500)):
        for keep in (0, 1, 700, 1499, 1500):
            run(t, 1500, 16, length, page(v), [keep])


def test_numbers_out_of_range():
    rng = np.random.default_rng(6)
    t = tables(rng, [20, 20], 20, 40)
    t[0, 3], t[1, 4] = 40, 2 ** 31 - 1            # no pages of the pool
    mass = rng.random((2, 2, 320)).astype(np.float32)
    for lens in ([2 ** 31 - 1, -5], [0, 1], [17, 10 ** 6]):
        run(t, 40, 16, lens, mass, [2, -(2 ** 31)], 0, 0)


def test_what_lies_behind_the_end_has_no_part():
    rng = np.random.default_rng(7)
    t = tables(rng, [10], 12, 12, holes=0.0)
    mass = rng.random((1, 2, 192)).astype(np.float32)
    a = run(t, 12, 16, [149], mass, [4])
    mass[..., 149:] = np.nan
    b = run(t, 12, 16, [149], mass, [4])
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_a_captured_eviction_replays():
    rng = np.random.default_rng(8)
    t = tables(rng, [400, 90], 400, 500)
    p = B.make_cache_params(2, 2, 64, page_tokens=16, n_pages=500, max_pages=400)
    td, lens, keep = torch.from_numpy(t).cuda(), i32([6400, 1440]), i32([100, 30])
    mass = torch.rand(2, 2, 6400, device="cuda")
    out = [torch.empty_like(td), torch.empty_like(td), torch.empty(2, dtype=torch.int32, device="cuda")]
    ws = B.alloc_ws(B.litevggt_cache_evict_ws_bytes(p))
    call = lambda o: B.litevggt_cache_evict(p, td, lens, mass, keep, 1, 1, *o, ws)      # noqa: E731
    call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out)
    for i in range(3):
        mass.copy_(torch.rand(2, 2, 6400, device="cuda"))
        keep.fill_(10 * i + 3)
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        call(out)
        assert all(torch.equal(a, b) for a, b in zip(got, out))


@pytest.mark.parametrize("dtype", ["e2m1", "bf16"])
def test_a_stream_in_a_bounded_pool(dtype):
    """Frames arrive: q and k are rotated by their rows and columns, k and v stored, the frame attends to what is held, what positions draw is
    added up, and pages leave so that the next frame has room.  The pool never grows; each step is checked against the plain one."""
    rng = np.random.default_rng(9)
    heads, dim, page, T, frames, budget = 2, 64, 16, 32, 7, 7
    columns, n_pages = frames * T // page, budget + T // page
    p = B.make_cache_params(1, heads, dim, cache_dtype=B.CACHE_E2M1 if dtype == "e2m1" else B.CACHE_BF16, page_tokens=page, n_pages=n_pages,
                            max_pages=columns, frame_tokens=T)
    turn = B.make_rope_params(heads, dim, (16, 16))
    cache, mass = B.alloc_cache(p), B.alloc_mass(p)
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None:
            x.zero_()
    table = np.full((1, columns), -1, np.int32)
    o = S.Cache4(n_pages, heads, page, dim, table) if dtype == "e2m1" else O.Cache(n_pages, heads, page, dim, table, False)
    free = list(range(n_pages))
    where = np.stack([np.arange(T) // 8 + 1, np.arange(T) % 8 + 1], 1).astype(np.int32)
    ws_a = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, T))
    ws_m = B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, T))
    ws_e = B.alloc_ws(B.litevggt_cache_evict_ws_bytes(p))
    freed, count = torch.empty(1, columns, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    for f in range(frames):
        for j in range(f * T // page, (f + 1) * T // page):
            table[0, j] = free.pop()
        cache.page_table.copy_(torch.from_numpy(table))
        q, k, v = (rows(rng, T, heads, dim) for _ in range(3))
        qd, kd = dev(q), dev(k)
        B.litevggt_rope(turn, torch.from_numpy(where).cuda(), qd, kd, qd, kd)
        off, length = i32([0, T]), i32([(f + 1) * T])
        B.litevggt_cache_write(p, cache, kd, dev(v), off, i32([f * T]))
        out = torch.empty(T, heads, dim, dtype=torch.bfloat16, device="cuda")
        B.litevggt_cached_attn(p, cache, qd, off, length, out, ws_a)
        before = host(mass)
        B.litevggt_cached_mass(p, cache, qd, off, length, mass, mass, ws_m)
        # the plain side goes on from the rotated rows, whose own test is elsewhere
        q, k = host(qd), host(kd)
        o.table = table
        o.write(k, v, [0, T], [f * T])
        want = O.cached_attention(o, q, [0, T], [(f + 1) * T], T)
        spread = np.abs(o.v).max()
        assert np.abs(host(out) - want).max() <= 2.0 ** -8 * np.abs(want).max() + (2.0 ** -8 + 2.0 ** -10) * spread
        drawn = S.mass(o, q, [0, T], [(f + 1) * T], T, before, before)
        assert np.abs(host(mass) - drawn).max() <= 2.0 ** -12 * drawn.max()
        exact = S.evict(table, n_pages, page, [(f + 1) * T], mass.cpu().numpy(), [budget - 0], 1, 1)
        B.litevggt_cache_evict(p, cache.page_table, length, mass, i32([budget]), 1, 1, cache.page_table, freed, count, ws_e)
        table = cache.page_table.cpu().numpy()
        assert np.array_equal(table, exact[0]) and np.array_equal(freed.cpu().numpy(), exact[1])
        free += freed[0, :int(count)].tolist()
        assert (table >= 0).sum() <= budget and len(free) + (table >= 0).sum() == n_pages
    assert (table >= 0).sum() == budget and table[0, 0] >= 0 and table[0, -1] >= 0


def test_more_columns_than_fit_beside_the_select():
    rng = np.random.default_rng(10)
    t = tables(rng, [17000, 20000], 20000, 40000)
    mass = rng.random((2, 1, 320000)).astype(np.float32)
    run(t, 40000, 16, [17000 * 16 - 5, 320000], mass, [9000, 19], 2, 2)
    run(t, 40000, 16, [17000 * 16 - 5, 320000], np.floor(mass * 3), [9000, 1900], 2, 2)


@pytest.mark.parametrize("heads,page", [(1, 16), (4, 16), (8, 16), (9, 16), (2, 64), (1, 128)])
def test_short_caches(heads, page):
    """Pages of few masses, which one kernel sums and selects, and the next sizes, which two do."""
    rng = np.random.default_rng(heads * page)
    for pages in ([1, 5, 0], [300, 1024], [1025]):
        t = tables(rng, pages, max(pages), sum(pages))
        lens = [max(0, c * page - int(rng.integers(0, page))) for c in pages]
        mass = np.floor(rng.random((len(pages), heads, max(pages) * page)) * 3).astype(np.float32)
        for s, n in enumerate(lens):
            mass[s, :, n:] = np.nan
        run(t, sum(pages), page, lens, mass, [c // 2 for c in pages], 0, 1)
        run(t, sum(pages), page, lens, mass, [c // 2 for c in pages], 1, 0, in_place=True)
