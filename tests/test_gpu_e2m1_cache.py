"""The E2M1 cache on the GPU: what is written, what is read back, attention over it, against the plain implementation in 64 bits.

Codes, scales and what is read back are exact.  Attention's tolerance: stream_cases.Pool.attend."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from oracle import stream_oracle as S
from paper_2512_04939_amd import binding as B

from stream_cases import Pool, dev, host, i32, packed, rows

pytestmark = pytest.mark.gpu


def same_pool(c):
    for name in ("k", "v"):
        assert np.array_equal(getattr(c.d, name).cpu().numpy(), packed(getattr(c.o, name + "c"))), name
        assert np.array_equal(getattr(c.d, name + "_scale").cpu().numpy(), (getattr(c.o, name + "e") + 127).astype(np.uint8)), name


@pytest.mark.parametrize("dim,heads,page,new,pos", [
    (64, 1, 16, [1], [0]), (64, 16, 64, [1], [500]), (64, 5, 16, [3, 0, 21, 1], [15, 7, 0, 40]), (128, 2, 32, [70, 5], [31, 0]),
    (64, 3, 1024, [70], [990]), (128, 4, 16, [2] * 70, list(range(70))),
])
def test_write_and_read(dim, heads, page, new, pos):
    c = Pool(1, [p + n for p, n in zip(pos, new)], heads=heads, kv_heads=heads, head_dim=dim, page=page, holes=[(0, 0)] if pos[0] > 20 else ())
    rng = np.random.default_rng(2)
    n = sum(new)
    off = [0] + np.cumsum(new).tolist()
    k, v = rows(rng, n + 2, heads, dim), rows(rng, n + 2, heads, dim, gain=30.0)
    if n > 2:
        k[1] = 0.0
        k[2, 0, 5], k[2, 0, 6] = np.inf, -np.inf
        v[0, 0, :4] = [2.0 ** -130, -2.0 ** 100, -0.0, 2.0 ** -126]
        v[1, 0, 33] = np.nan
    both = dev(np.concatenate([k.reshape(n + 2, -1), v.reshape(n + 2, -1)], 1))
    kd, vd = both[:, :heads * dim].unflatten(1, (heads, dim)), both[:, heads * dim:].unflatten(1, (heads, dim))
    B.litevggt_cache_write(c.p, c.d, kd, vd, i32(off), i32(pos))
    c.o.write(k, v, off, pos)
    same_pool(c)
    out = [torch.full((n + 2, heads, dim), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.litevggt_cache_read(c.p, c.d, i32(pos), i32(off), *out)
    for j in range(2):
        got = host(out[j])
        assert (got[n:] == 5.0).all()
        for s in range(len(new)):
            want = c.o.rows(s, pos[s], new[s])[j]
            assert np.array_equal(got[off[s]:off[s + 1]], want, equal_nan=True)


def test_every_bf16_value_rounds_as_defined():
    """All finite values, each in a block whose largest is itself, 6 times, and 2.4 times as large."""
    bits = np.arange(65536, dtype=np.uint32)
    x = (bits << 16).view(np.float32)
    x = x[np.isfinite(x)].astype(np.float64)
    with np.errstate(over="ignore"):
        tops = np.stack([x, O.round_bf16(x * 6), O.round_bf16(x * 2.4)])
    tops = np.where(np.abs(tops) > 3.3e38, x, tops)
    block = np.zeros((3, len(x), 32))
    block[..., 0], block[..., 31], block[..., 17] = tops, x, -x
    block = block.reshape(-1, 1, 64)
    n = len(block)
    p = B.make_cache_params(1, 1, 64, cache_dtype=B.CACHE_E2M1, page_tokens=1024, n_pages=-(-n // 1024), max_pages=-(-n // 1024))
    c = B.alloc_cache(p)
    c.page_table.copy_(torch.arange(p.max_pages, device="cuda").int()[None])
    kd = dev(block)
    B.litevggt_cache_write(p, c, kd, kd, i32([0, n]), i32([0]))
    flat = block.reshape(-1, 32)
    top = np.abs(flat).max(1)
    e = np.where(top > 0, np.frexp(top)[1] - 5, 0)
    for _ in range(3):
        e = np.where((top > 0) & (top > 6.0 * 2.0 ** e.astype(float)), e + 1, e)
    e = np.maximum(e, -126)
    z = flat[:, [0, 17, 31]] / 2.0 ** e[:, None].astype(float)
    grid = np.array(S.E2M1)
    dist = np.abs(np.abs(z)[..., None] - grid)
    best = dist.min(-1, keepdims=True)
    even = np.where(dist == best, np.arange(8) % 2, 9).argmin(-1)
    code = even | np.where(np.signbit(z), 8, 0)
    for codes, scales in ((c.k, c.k_scale), (c.v, c.v_scale)):
        got = codes.cpu().numpy().reshape(-1, 16)[:len(flat)]
        assert np.array_equal(scales.cpu().numpy().reshape(-1)[:len(flat)], (e + 127).astype(np.uint8))
        assert np.array_equal(got[:, 0] & 15, code[:, 0]) and np.array_equal(got[:, 8] >> 4, code[:, 1]) and np.array_equal(got[:, 15] >> 4, code[:, 2])
    out = [torch.empty(n, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.litevggt_cache_read(p, c, i32([0]), i32([0, n]), *out)
    got = host(out[0]).reshape(-1, 32)[:, [0, 17, 31]]
    with np.errstate(over="ignore"):
        want = O.round_bf16(np.copysign(grid[even], z) * 2.0 ** e[:, None].astype(float))
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(got, want)


def test_norm_is_applied_before_rounding():
    c = Pool(3, [40], heads=2, kv_heads=2, qk_norm=1)
    rng = np.random.default_rng(4)
    k, v = rows(rng, 40, 2, 64, gain=7.0), rows(rng, 40, 2, 64)
    B.litevggt_cache_write(c.p, c.d, dev(k), dev(v), i32([0, 40]), i32([0]))
    c.o.write(k, v, [0, 40], [0], qk_norm=True)
    got = c.d.k.cpu().numpy()
    # a value on the border of two bf16 values may fall to the other side in 32 bits: 40 * 128 values, one in 2^10 of these at most near a border
    assert (got != packed(c.o.kc)).sum() <= 5 and np.array_equal(c.d.v.cpu().numpy(), packed(c.o.vc))


FORMS = [
    dict(lens=[1], new=[1]), dict(lens=[394], new=[1], page=64, frame=1), dict(lens=[130], new=[5], heads=4, kv_heads=2, page=32),
    dict(lens=[301, 1, 0, 77], new=[1, 1, 0, 3], heads=8, kv_heads=2, head_dim=128, frame=1),
    dict(lens=[200, 63], new=[40, 63], heads=4, kv_heads=4, frame=9), dict(lens=[700], new=[300], heads=2, kv_heads=1, frame=50, page=32),
    dict(lens=[700, 90], new=[300, 90], heads=4, kv_heads=2, frame=1, head_dim=128), dict(lens=[2600], new=[2], heads=2, kv_heads=2, page=16),
    dict(lens=[2600], new=[40], heads=2, kv_heads=2, page=16, head_dim=128, frame=13), dict(lens=[1300], new=[600], heads=2, kv_heads=2),
    dict(lens=[33] * 70, new=[1] * 70, heads=2, kv_heads=2, frame=1),
]


@pytest.mark.parametrize("holes", [False, True])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_attention(form, holes):
    form = dict(form)
    lens, new = form.pop("lens"), form.pop("new")
    page = form.get("page", 16)
    gone = [(s, c) for s, n in enumerate(lens) for c in range(-(-n // page)) if c % 3 == 1] if holes else ()
    Pool(5, lens, holes=gone, **form).attend(new, tail=2)


@pytest.mark.parametrize("dim,new", [(64, 1), (64, 40), (64, 200), (128, 3), (128, 90)])
def test_what_is_not_seen_has_no_part(dim, new):
    """NaN blocks behind the last position, in positions that no query may see, and in a page that is not held."""
    c = Pool(6, [260], heads=2, kv_heads=2, head_dim=dim, page=16, frame=20, holes=[(0, 3)], more_columns=1)
    got = c.attend([new])
    t = c.table[0]
    for s in (c.d.k_scale, c.d.v_scale):
        s[int(t[260 // 16]), :, 260 % 16:] = 255
        for j in set(range(c.n_pages)) - set(t[t >= 0].tolist()):
            s[j] = 255
    q = rows(np.random.default_rng(7), new, 2, dim)
    a = c.attend([new], q=q)
    assert np.isfinite(got).all() and np.isfinite(a).all()


@pytest.mark.parametrize("dim,new", [(64, 3), (64, 150), (128, 3), (128, 100)])
def test_nan_where_a_row_sees_it(dim, new):
    c = Pool(8, [250], heads=1, kv_heads=1, head_dim=dim, page=16, frame=10)
    page, row = int(c.table[0, 240 // 16]), 240 % 16
    c.o.v[page, 0, row, :32] = np.nan
    c.d.v_scale[page, 0, row, 0] = 255
    got = c.attend([new])
    assert np.isnan(got[-10:, 0, :32]).all() and np.isfinite(got[..., 32:]).all() and np.isfinite(got[:max(0, new - 10)]).all()


def test_large_scales_and_scores():
    Pool(9, [300], heads=2, kv_heads=2, gain=64.0).attend([3])
    Pool(9, [300], heads=2, kv_heads=2, gain=64.0).attend([120])
    Pool(10, [300], heads=2, kv_heads=2, head_dim=128, scale=0.5).attend([7])


def test_captured_write_and_attention_replay_with_other_lengths():
    c = Pool(11, [200, 150], heads=4, kv_heads=2, page=16, frame=1)
    p = c.p
    rng = np.random.default_rng(12)
    k, v, q = rows(rng, 2, 2, 64), rows(rng, 2, 2, 64), rows(rng, 2, 4, 64)
    kd, vd, qd = dev(k), dev(v), dev(q)
    off, pos, length = i32([0, 1, 2]), i32([10, 20]), i32([11, 21])
    o = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, 2))

    def step():
        B.litevggt_cache_write(p, c.d, kd, vd, off, pos)
        B.litevggt_cached_attn(p, c.d, qd, off, length, o, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for at in ([30, 21], [199, 149], [0, 5]):
        pos.copy_(i32(at))
        length.copy_(i32([x + 1 for x in at]))
        o.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        got = o.clone()
        o.fill_(9.0)
        step()
        assert torch.equal(got, o)


def test_calls_on_two_streams_at_once():
    c = Pool(13, [500, 300], heads=4, kv_heads=4, frame=1)
    rng = np.random.default_rng(14)
    q = [dev(rows(rng, 2, 4, 64)) for _ in range(2)]
    off, length = i32([0, 1, 2]), i32([500, 300])
    want = [torch.empty_like(x) for x in q]
    got = [torch.empty_like(x) for x in q]
    ws = [B.alloc_ws(B.litevggt_cached_attn_ws_bytes(c.p, 2)) for _ in range(2)]
    for i in range(2):
        B.litevggt_cached_attn(c.p, c.d, q[i], off, length, want[i], ws[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                B.litevggt_cached_attn(c.p, c.d, q[i], off, length, got[i], ws[i])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
