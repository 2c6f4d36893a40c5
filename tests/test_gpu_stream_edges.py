"""Calls at the edges of what the documentation allows: more queries than positions, lengths beyond the table, huge frames, pools over 4 GB, for
attention over an E2M1 cache and for the weight that positions draw (tolerances: stream_cases)."""
import numpy as np
import pytest
import torch

from oracle import stream_oracle as S
from paper_2512_04939_amd import binding as B

from stream_cases import Pool, dev, host, i32, packed, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frame", [0, 1, 4, 2 ** 31 - 1])
@pytest.mark.parametrize("lens,new", [([5], [9]), ([40, 3], [41, 200]), ([100], [130]), ([0], [3]), ([17, 33, 31], [1, 2, 3])], ids=str)
def test_more_queries_than_positions_and_frames_of_any_size(lens, new, frame):
    for dim, dtype in ((64, "e2m1"), (128, "e2m1"), (64, "bf16")):
        c = Pool(41, lens, heads=4, kv_heads=2, head_dim=dim, dtype=dtype, frame=frame)
        c.attend(new)
        c.draw(new)


@pytest.mark.parametrize("new", [1, 70])
def test_lengths_beyond_the_table(new):
    c = Pool(42, [64, 64], heads=2, kv_heads=2, dtype="e2m1", frame=3)
    for length in ([70, 64], [64, 5000], [65, 10 ** 9]):
        c.attend([new, new], kv_len=length)
        c.draw([new, new], kv_len=length)


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("length", [1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 255, 257])
def test_every_kind_of_last_tile(length, page):
    for dim in (64, 128):
        c = Pool(43, [length], heads=2, kv_heads=1, head_dim=dim, page=page)
        # what lies behind the end is NaN
        t, at = c.table[0], length % page
        if at:
            for s in (c.d.k_scale, c.d.v_scale):
                s[int(t[length // page]), :, at:] = 255
        c.attend([1])
        c.draw([1])
        c.attend([min(length, 40)])
        c.draw([min(length, 40)])


@pytest.mark.parametrize("dim", [64, 128])
def test_pools_over_4_gb(dim):
    """Pages whose bytes begin beyond 2^32 in both pools, and below."""
    page, heads = 1024, 16
    n_pages = (1 << 32) // (page * heads * dim // 2) + 40
    lens = [3 * page + 100]
    small = Pool(44, lens, heads=heads, kv_heads=heads, head_dim=dim, page=page)
    p = B.make_cache_params(1, heads, dim, cache_dtype=B.CACHE_E2M1, page_tokens=page, n_pages=n_pages, max_pages=small.max_pages)
    big = B.CacheBuffers(*(torch.empty(n_pages, heads, page, dim // 2, dtype=torch.uint8, device="cuda") for _ in range(2)),
                         *(torch.empty(n_pages, heads, page, dim // 32, dtype=torch.uint8, device="cuda") for _ in range(2)), None)
    where = [n_pages - 1, 3, n_pages - 7, 0]
    for j, to in enumerate(where):
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(big, name)[to] = getattr(small.d, name)[int(small.table[0, j])]
    big.page_table = torch.tensor([where], dtype=torch.int32, device="cuda")
    for new in (2, 90):
        q = dev(rows(np.random.default_rng(1), new, heads, dim))
        outs, masses = [], []
        for params, cache in ((small.p, small.d), (p, big)):
            o = torch.empty_like(q)
            B.litevggt_cached_attn(params, cache, q, i32([0, new]), i32(lens), o, B.alloc_ws(B.litevggt_cached_attn_ws_bytes(params, new)))
            m = B.alloc_mass(params)
            B.litevggt_cached_mass(params, cache, q, i32([0, new]), i32(lens), None, m, B.alloc_ws(B.litevggt_cached_mass_ws_bytes(params, new)))
            outs.append(o)
            masses.append(m)
        assert torch.equal(outs[0], outs[1]) and torch.equal(masses[0], masses[1])
    k = dev(rows(np.random.default_rng(2), 200, heads, dim))
    B.litevggt_cache_write(p, big, k, k, i32([0, 200]), i32([900]))
    back = [torch.empty_like(k) for _ in range(2)]
    B.litevggt_cache_read(p, big, i32([900]), i32([0, 200]), *back)
    want = S.round_blocks(host(k[::37]))[0]
    assert np.array_equal(host(back[0][::37]), want) and torch.equal(*back)


def test_rows_of_no_sequence_are_left_out():
    """Tokens between and behind the sequences' rows."""
    c = Pool(45, [100, 50], heads=2, kv_heads=2, dtype="e2m1", frame=1)
    q = rows(np.random.default_rng(3), 20, 2, 64)
    q[4:9], q[12:] = np.nan, np.nan
    p = c.p
    got = B.alloc_mass(p)
    ws = B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, 20)).fill_(255)
    B.litevggt_cached_mass(p, c.d, dev(q), i32([9, 12, 12]), i32([100, 50]), None, got, ws)
    want = S.mass(c.o, q, [9, 12, 12], [100, 50], 1, None, np.zeros(tuple(got.shape)))
    assert torch.isfinite(got).all() and np.abs(host(got) - want).max() <= 2.0 ** -14 and np.abs(want).sum() > 5


def test_two_graphs_with_workspaces_of_their_own():
    c = Pool(46, [300, 200], heads=4, kv_heads=2, dtype="e2m1", frame=1)
    p = c.p
    q = [dev(rows(np.random.default_rng(i), 6, 4, 64)) for i in range(2)]
    off, length = i32([0, 3, 6]), i32([300, 200])
    out = [B.alloc_mass(p) for _ in range(2)]
    ws = [B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, 6)) for _ in range(2)]
    call = lambda i, o: B.litevggt_cached_mass(p, c.d, q[i], off, length, None, o, ws[i])      # noqa: E731
    graphs = []
    for i in range(2):
        call(i, out[i])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, out[i])
        graphs.append(g)
    want = [x.clone() for x in out]
    for _ in range(3):
        for i in (1, 0):
            out[i].fill_(7)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(out[i][0, :, :300], want[i][0, :, :300]) and torch.equal(out[i][1, :, :200], want[i][1, :, :200])
