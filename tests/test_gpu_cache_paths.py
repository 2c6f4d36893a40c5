"""Attention over the paged cache and cross attention at sizes where their keys are cut, lists of pages are walked and sequences are
many, against the softmax written out in 64 bits (torch, on the GPU).

Tolerances: a weight is rounded to bf16 for the second product and so is the result (each off by at most 2^-8 of itself);
a score is a sum of d products in fp32, off by at most d 2^-24 of sum |q k| <= d max|q| max|k|, and an exponent's error is that share of
a weight.  So |got - o| <= 2^-8 |o| + (2^-8 + 4 scale d^2 2^-24 max|q| max|k|) sum w |v| / sum w (twice for the sum of
weights, twice for the exponential's own)."""
import numpy as np
import pytest
import torch

from paper_2512_04939_amd import binding as B

pytestmark = pytest.mark.gpu


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)


def gen_of(seed):
    return torch.Generator("cuda").manual_seed(seed)


def i32(x):
    return torch.tensor([int(y) for y in x], dtype=torch.int32, device="cuda")


def plain(q, k, v, see):
    """q [n, h, d], k, v [m, kv, d], see [n, m] bool; (output, sum w |v| / sum w, bound), float64.  Values of V that a query does not
    see have no part; one that sees nothing gives zeros."""
    n, h, d = q.shape
    group, scale = h // k.shape[1], d ** -0.5
    out = torch.zeros(n, h, d, dtype=torch.float64, device=q.device)
    spread = torch.zeros_like(out)
    for j in range(h):
        kk, vv = k[:, j // group].double(), v[:, j // group].double()
        wild = ~torch.isfinite(kk).all(1) | ~torch.isfinite(vv).all(1)
        assert not (see & wild).any()
        kk, vv = torch.where(wild[:, None], 0.0, kk), torch.where(wild[:, None], 0.0, vv)
        s = (q[:, j].double() @ kk.T.contiguous() * scale).masked_fill(~see, -torch.inf)
        w = torch.nan_to_num(torch.softmax(s, 1), nan=0.0)
        out[:, j], spread[:, j] = w @ vv, w @ vv.abs()
    km = torch.where(torch.isfinite(k), k.double(), 0.0).abs().max() if k.numel() else 0.0
    score = 4 * scale * d * d * 2.0 ** -24 * q.double().abs().max() * km
    return out, 2.0 ** -8 * out.abs() + (2.0 ** -8 + score) * spread + 1e-30


def near(got, out, tol):
    assert torch.isfinite(got).all()
    bad = (got.double() - out).abs() > tol
    assert not bad.any(), (bad.nonzero()[:5].tolist(), ((got.double() - out).abs() / tol).max().item())


class Paged:
    def __init__(self, seed, lens, *, heads, kv_heads, dim, e4m3=False, page=16, frame=0, lost=0.0, table=None):
        self.gen, self.lens, self.frame, self.e4m3, self.page = gen_of(seed), list(lens), frame, e4m3, page
        rng = np.random.default_rng(seed)
        pages = [-(-n // page) for n in lens]
        most = max(pages + [1])
        n_pages = sum(pages) + 2
        if table is None:
            ids = rng.permutation(n_pages)
            table = np.full((len(lens), most), -1, np.int32)
            at = 0
            for s, c in enumerate(pages):
                table[s, :c] = ids[at:at + c]
                at += c
            table[rng.random(table.shape) < lost] = -1
        self.table = table
        self.p = B.make_cache_params(len(lens), heads, dim, kv_heads=kv_heads, cache_dtype=B.CACHE_E4M3 if e4m3 else B.CACHE_BF16,
                                     page_tokens=page, n_pages=n_pages, max_pages=table.shape[1], frame_tokens=frame)
        self.c = B.alloc_cache(self.p)
        self.c.page_table.copy_(torch.from_numpy(np.ascontiguousarray(table)))
        for x in (self.c.k, self.c.v):
            y = randn(self.gen, *x.shape)
            x.copy_((y.float() * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if e4m3 else y)
        if e4m3:
            for x in (self.c.k_scale, self.c.v_scale):
                x.copy_(torch.randint(119, 122, x.shape, generator=self.gen, device="cuda"))

    def rows(self, s, name):
        """Positions of sequence s, [len, kv, d] float64, and which of them are held."""
        t = torch.from_numpy(self.table[s].astype(np.int64)).cuda()
        pos = torch.arange(self.lens[s], device="cuda")
        held = t[pos // self.page] >= 0
        x = getattr(self.c, name)
        if self.e4m3:
            e = getattr(self.c, name + "_scale").double() - 127
            x = x.view(torch.float8_e4m3fn).double() * torch.exp2(e)[..., None]
        return x[t[pos // self.page].clamp(min=0), :, pos % self.page], held

    def see(self, s, n):
        """[n, len] bool: what the last n positions' queries see"""
        pos = torch.arange(self.lens[s], device="cuda")
        at = self.lens[s] - n + torch.arange(n, device="cuda")
        if self.frame:
            return pos[None] < ((torch.div(at, self.frame, rounding_mode="floor") + 1) * self.frame * (at >= 0))[:, None]
        return torch.ones(n, self.lens[s], dtype=torch.bool, device="cuda")

    def run(self, q, new, o=None, ws=None):
        off = np.concatenate([[0], np.cumsum(new)])
        o = torch.full_like(q, 7.0) if o is None else o
        ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(self.p, len(q))) if ws is None else ws
        B.litevggt_cached_attn(self.p, self.c, q, i32(off), i32(self.lens), o, ws)
        return o

    def check(self, new, some=None):
        """All sequences, or `some` of them, of a call of new[s] tokens each."""
        q = randn(self.gen, int(sum(new)), self.p.heads, self.p.head_dim)
        got = self.run(q, new)
        off = np.concatenate([[0], np.cumsum(new)])
        for s in range(len(new)) if some is None else some:
            a, b = int(off[s]), int(off[s + 1])
            if a == b:
                continue
            if self.lens[s] == 0:
                assert not got[a:b].any()
                continue
            (k, held), (v, _) = self.rows(s, "k"), self.rows(s, "v")
            near(got[a:b], *plain(q[a:b], k, v, self.see(s, b - a) & held))
        return got


def cross(q, k, v, q_off, begin, end, ws=None):
    p = B.make_cross_params(len(begin), q.shape[1], q.shape[2], kv_heads=k.shape[1])
    o = torch.full_like(q, 7.0)
    ws = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, len(q), len(k))) if ws is None else ws
    ws.fill_(255)
    B.litevggt_cross_attn(p, q, i32(q_off), k, v, i32(begin), i32(end), o, ws)
    return o


# one sequence whose blocks of 256 rows fill the chip's slots once and a few more: the first heads' are not cut, the others' are
@pytest.mark.parametrize("dim,kv,group,n,m", [(64, 12, 1, 11013, 701), (128, 6, 1, 11013, 701), (64, 3, 4, 11001, 1500), (128, 3, 3, 7500, 1023)])
def test_one_sequence_of_more_blocks_than_slots(dim, kv, group, n, m):
    g = gen_of(n)
    q, k, v = randn(g, n, kv * group, dim), randn(g, m, kv, dim), randn(g, m, kv, dim)
    o = cross(q, k, v, [0, n], [0], [m])
    near(o, *plain(q, k, v, torch.ones(n, m, dtype=torch.bool, device="cuda")))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_frames_of_one_sequence_of_more_blocks_than_slots(dim, e4m3):
    n = 11013
    Paged(1, [n + 37], heads=12, kv_heads=12, dim=dim, e4m3=e4m3, frame=1041).check([n])


# pieces of more than 61 stages, of more than 256 groups of 16, some of whose pages are not held
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lost,page,frame", [(0.0, 16, 0), (0.3, 16, 0), (0.9, 16, 0), (0.2, 128, 700), (0.97, 32, 0)])
def test_long_lists_of_pages(lost, page, frame, dim, e4m3):
    Paged(2, [20000], heads=16, kv_heads=16, dim=dim, e4m3=e4m3, page=page, frame=frame, lost=lost).check([2048])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("new", [1, 40, 100])
def test_no_page_held(new, e4m3):
    c = Paged(3, [5000, 300], heads=4, kv_heads=2, dim=64, e4m3=e4m3, lost=2.0)
    assert not c.check([new, new]).any()


# more than 64 sequences, a few of them long enough to be cut, empty ones between
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_seq,new,frame", [(150, 1, 0), (150, 3, 1), (70, 45, 0), (66, 130, 1), (200, 70, 16)])
def test_many_sequences(n_seq, new, frame, dim, e4m3):
    rng = np.random.default_rng(n_seq + new)
    lens = rng.integers(0, 300, n_seq)
    lens[[3, 65]] = [9000, 7777]
    news = np.minimum(rng.integers(0, 2 * new + 1, n_seq), lens)
    news[[3, 65]] = new
    Paged(4, lens, heads=4, kv_heads=2, dim=dim, e4m3=e4m3, page=32, frame=frame, lost=0.05).check(news)


@pytest.mark.parametrize("n_seq", [65, 1000, 4096, 4097, 9000])
def test_thousands_of_sequences(n_seq):
    rng = np.random.default_rng(n_seq)
    lens = rng.integers(0, 40, n_seq)
    lens[[1, n_seq - 1]] = [2500, 1111]
    news = np.minimum(rng.integers(0, 3, n_seq), lens)
    news[[1, n_seq - 1]] = 2
    some = [0, 1, 63, 64, n_seq // 2, n_seq - 2, n_seq - 1] + rng.integers(0, n_seq, 40).tolist()
    Paged(17, lens, heads=2, kv_heads=1, dim=64, page=16, lost=0.02).check(news, some)
    Paged(18, lens, heads=40, kv_heads=1, dim=128, e4m3=True, page=16, frame=1).check(news, some)


@pytest.mark.parametrize("n_seq", [64, 65, 4097])
def test_write_and_read_of_many_sequences(n_seq):
    """What is written comes back; rows of no sequence are left alone on both sides."""
    g, rng = gen_of(n_seq), np.random.default_rng(n_seq)
    new = rng.integers(0, 4, n_seq)
    pos = rng.integers(0, 30, n_seq)
    first, n = 3, int(new.sum())      # (three rows before the first sequence's, four behind the last)
    p = B.make_cache_params(n_seq, 2, 64, page_tokens=16, n_pages=3 * n_seq, max_pages=3)
    c = B.alloc_cache(p)
    c.page_table.copy_(torch.from_numpy(rng.permutation(3 * n_seq).reshape(n_seq, 3).astype(np.int32)))
    off = i32(first + np.concatenate([[0], np.cumsum(new)]))
    k, v = randn(g, n + 7, 2, 64), randn(g, n + 7, 2, 64)
    c.k.zero_()
    B.litevggt_cache_write(p, c, k, v, off, i32(pos))
    assert int((c.k != 0).any(-1).any(1).sum()) == n
    a, b = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    B.litevggt_cache_read(p, c, i32(pos), off, a, b)
    assert torch.equal(a[first:first + n], k[first:first + n]) and torch.equal(b[first:first + n], v[first:first + n])
    assert (a[:first] == 7.0).all() and (b[first + n:] == 7.0).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv", [(7, 1), (15, 5), (14, 2), (1, 1)])
@pytest.mark.parametrize("new", [1, 5, 37, 90, 300])
def test_odd_heads(new, heads, kv, dim):
    Paged(5, [new + 1500, new, new + 131], heads=heads, kv_heads=kv, dim=dim, frame=1).check([new, new, new])


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [2, 50, 400])
def test_wild_values_behind_the_frame_of_a_query(new, dim, e4m3):
    """The last frame's rows are infinities and NaN; all rows but its own see none of it."""
    frame, length = 130, 1300
    c = Paged(6, [length], heads=4, kv_heads=4, dim=dim, e4m3=e4m3, frame=frame)
    pages = c.c.page_table[0].long()
    pos = torch.arange(length - 65, length, device="cuda")
    for x in (c.c.k, c.c.v):
        if e4m3:
            x[pages[pos // 16], :, pos % 16] = 0x7F          # NaN
        else:
            x[pages[pos // 16], :, pos % 16] = torch.tensor([torch.inf, torch.nan, -torch.inf, 1.0] * (dim // 4), device="cuda").to(torch.bfloat16)
    # the queries' own positions end a frame before the wild one
    q = randn(c.gen, new, 4, dim)
    o = torch.full_like(q, 7.0)
    off, ends = i32([0, new]), i32([length - frame])
    B.litevggt_cached_attn(c.p, c.c, q, off, ends, o, B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, new)))
    clean = Paged(6, [length], heads=4, kv_heads=4, dim=dim, e4m3=e4m3, frame=frame)
    clean.lens = [length - frame]
    (k, held), (v, _) = clean.rows(0, "k"), clean.rows(0, "v")
    near(o, *plain(q, k, v, clean.see(0, new) & held))
    # a longer sequence: the rows of the frames before the last keep clear of it
    n = new + frame
    q = torch.cat([q, randn(c.gen, frame, 4, dim)])
    got = c.run(q, [n])
    c.lens = [length - 65]
    (k, held), (v, _) = c.rows(0, "k"), c.rows(0, "v")
    see = clean.see(0, new)
    near(got[:new], *plain(q[:new], k[:length - frame], v[:length - frame], see & held[:length - frame]))
    assert torch.isnan(got[new:]).any()


def test_values_as_large_as_allowed():
    g = gen_of(7)
    for n in (3, 50, 300):
        q, k, v = randn(g, n, 2, 64), randn(g, 900, 2, 64), randn(g, 900, 2, 64)
        q[:, :, 0] = 20.0
        k[:, :, 0] = torch.arange(900, device="cuda")[:, None] * 0.01      # weights that grow along the axis
        v = v * 2.0 ** 77                                              # (none of N(0, 1) here is beyond 8)
        o = cross(q, k, v, [0, n], [0], [900])
        near(o, *plain(q, k, v, torch.ones(n, 900, dtype=torch.bool, device="cuda")))


def test_rows_that_lie_far_apart():
    """Strides of 2^26 elements: 128 MB from row to row, the last ones beyond 4 GB."""
    m, d = 37, 64
    pool = torch.empty(m << 26, dtype=torch.bfloat16, device="cuda")
    g = gen_of(8)
    for n in (2, 40, 130):
        far = pool.as_strided((m, 4 * d), (1 << 26, 1))
        far.copy_(randn(g, m, 4 * d))
        k, v = far[:, :2 * d].unflatten(1, (2, d)), far[:, 2 * d:].unflatten(1, (2, d))
        q = randn(g, n, 2, d)
        o = cross(q, k, v, [0, n], [0], [m])
        near(o, *plain(q, k, v, torch.ones(n, m, dtype=torch.bool, device="cuda")))


def test_a_page_that_serves_twice():
    """Two sequences over the same pages, one page at two places of a sequence."""
    table = np.array([[0, 1, 2, 1], [2, 1, 0, 0]], np.int32)
    for new in (1, 20, 60):
        Paged(9, [64, 55], heads=4, kv_heads=4, dim=64, table=table).check([new, min(new, 55)])


@pytest.mark.parametrize("new", [1, 40, 200])
def test_padded_batch(new):
    """Sequences at a fixed stride in q, k and v with other lengths: offsets name the rows that are there, the padding is left as it was."""
    g = gen_of(10)
    n_seq, m, h, d = 5, 400, 4, 64
    lens, news = [400, 1, 0, 333, 64], [new, 1, new, 0, max(new - 1, 1)]
    q, k, v = randn(g, n_seq * new, h, d), randn(g, n_seq * m, h, d), randn(g, n_seq * m, h, d)
    # (offsets ascend by sequence: rows between two sequences' are given a sequence without keys, which reads zeros)
    q_off, begin, end = [0], [], []
    for s in range(n_seq):
        q_off += [s * new + news[s], (s + 1) * new]
        begin += [s * m, 0]
        end += [s * m + lens[s], 0]
    o = cross(q, k, v, q_off, begin, end)
    for s in range(n_seq):
        a, n = s * new, news[s]
        see = torch.ones(n, lens[s], dtype=torch.bool, device="cuda")
        if n and lens[s]:
            near(o[a:a + n], *plain(q[a:a + n], k[s * m:s * m + lens[s]], v[s * m:s * m + lens[s]], see))
        elif n:
            assert not o[a:a + n].any()
        assert not o[a + n:a + new].any()


def test_scratch_of_a_longer_call_serves_the_shorter():
    c = Paged(11, [900] * 40, heads=8, kv_heads=8, dim=64)
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, 40 * 600))
    for new in (1, 20, 50, 100, 400, 600):
        q = randn(c.gen, 40 * new, 8, 64)
        assert torch.equal(c.run(q, [new] * 40, ws=ws), c.run(q, [new] * 40))


def test_two_streams_with_scratch_of_their_own():
    cs = [Paged(12 + i, [30000, 4000], heads=4, kv_heads=4, dim=64, e4m3=bool(i)) for i in range(2)]
    qs = [randn(c.gen, 2 * n, 4, 64) for c, n in zip(cs, (1, 150))]
    news = [[1, 1], [150, 150]]
    want = [c.run(q, n) for c, q, n in zip(cs, qs, news)]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = [[], []]
    spaces = [B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, len(q))) for c, q in zip(cs, qs)]
    outs = [[torch.full_like(q, 7.0) for _ in range(5)] for q in qs]
    args = [(i32(np.concatenate([[0], np.cumsum(n)])), i32(c.lens)) for c, n in zip(cs, news)]
    torch.cuda.synchronize()
    for r in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                B.litevggt_cached_attn(cs[i].p, cs[i].c, qs[i], *args[i], outs[i][r], spaces[i])
                got[i].append(outs[i][r])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


@pytest.mark.parametrize("new", [1, 40, 300])
def test_a_cut_call_captured_and_replayed_between_eager_ones(new):
    c = Paged(14, [9000, 500], heads=4, kv_heads=4, dim=128, e4m3=True)
    q, off = randn(c.gen, 2 * new, 4, 128), i32([0, new, 2 * new])
    ends, o = i32([9000, 500]), torch.zeros(2 * new, 4, 128, dtype=torch.bfloat16, device="cuda")
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, 2 * new))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.litevggt_cached_attn(c.p, c.c, q, off, ends, o, ws)
    for lens in ([9000, 500], [700, 500], [1, 0], [2500, 2500], [9000, 500]):
        lens = [min(x, y) for x, y in zip(lens, [9000, 500])]
        ends.copy_(i32(lens))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c.lens = lens
        assert torch.equal(o, c.run(q, [new, new]))


def test_a_captured_cross_attention_over_growing_states():
    g = gen_of(15)
    m, n = 6000, 300
    q, k, v = randn(g, n, 4, 64), randn(g, m, 4, 64), randn(g, m, 4, 64)
    p = B.make_cross_params(1, 4, 64, qk_norm=1)
    ws, other = (B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, n, m)) for _ in range(2))
    off, begin, end, o = i32([0, n]), i32([0]), i32([10]), torch.zeros_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.litevggt_cross_attn(p, q, off, k, v, begin, end, o, ws)
    for length in (10, 6000, 65, 0, 3001):
        end.fill_(length)
        graph.replay()
        eager = torch.empty_like(q)
        B.litevggt_cross_attn(p, q, off, k, v, begin, end, eager, other)
        torch.cuda.synchronize()
        assert torch.equal(o, eager)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [20, 50, 400])
def test_a_query_that_is_not_finite_keeps_to_itself(n, dim):
    g = gen_of(16)
    q, k, v = randn(g, n, 2, dim), randn(g, 1500, 2, dim), randn(g, 1500, 2, dim)
    bad = [0, 7, n - 1]
    hurt = q.clone()
    hurt[bad[0]], hurt[bad[1], 0, 3], hurt[bad[2]] = torch.nan, torch.inf, -torch.inf
    o = cross(hurt, k, v, [0, n], [0], [1500])
    out, tol = plain(q, k, v, torch.ones(n, 1500, dtype=torch.bool, device="cuda"))
    fine = torch.ones(n, 2, dtype=torch.bool, device="cuda")
    fine[[0, 0, 7, n - 1, n - 1], [0, 1, 0, 0, 1]] = False
    near(o[fine], out[fine], tol[fine])
    assert not torch.isfinite(o[~fine]).any()


def test_first_call_of_a_process_is_captured():
    """Nothing that a first call sets up may disturb a capture."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2512_04939_amd import binding as B
g = torch.Generator("cuda").manual_seed(1)
q, k, v = (torch.randn(n, 4, 64, generator=g, device="cuda").to(torch.bfloat16) for n in (300, 3000, 3000))
off, begin, end = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 300], [0], [3000]))
p = B.make_cross_params(1, 4, 64)
o, eager = torch.zeros_like(q), torch.zeros_like(q)
ws = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, 300, 3000))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    B.litevggt_cross_attn(p, q, off, k, v, begin, end, o, ws)
for _ in range(3):
    o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    B.litevggt_cross_attn(p, q, off, k, v, begin, end, eager, ws)
    torch.cuda.synchronize()
    assert eager.any() and torch.equal(o, eager)
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
