"""Offsets that do not ascend, lengths and page numbers of any value: no call leaves the sizes in its parameters.  What the rows in between
come to is not defined; rows behind them, and pages beyond the pool, stay as they were."""
import numpy as np
import pytest
import torch

from paper_2512_04939_amd import binding as B

pytestmark = pytest.mark.gpu
BEHIND = 300


def i32(x):
    return torch.from_numpy(np.asarray(x, np.int64).astype(np.int32)).cuda()


def randn(*shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)


def numbers(rng, n, most, kind):
    """n numbers: of all sizes, of the sizes of the call, or all and nothing in turn"""
    if kind == "any":
        return rng.integers(-2 ** 31, 2 ** 31, n)
    if kind == "near":
        return rng.integers(-3, most + 4, n)
    return np.arange(n) % 2 * most


@pytest.mark.parametrize("kind", ["any", "near", "turns"])
@pytest.mark.parametrize("n_seq,n", [(2, 400), (60, 50), (64, 9000), (65, 60), (500, 300), (1100, 40000)])
def test_cross_attention(n_seq, n, kind):
    rng = np.random.default_rng(n_seq)
    for dim, m in ((64, 3000), (128, 700)):
        q, k, v = randn(n, 4, dim), randn(m, 2, dim), randn(m, 2, dim)
        o = torch.full((n + BEHIND, 4, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        p = B.make_cross_params(n_seq, 4, dim, kv_heads=2)
        ws = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, n, m)).fill_(255)
        B.litevggt_cross_attn(p, q, i32(numbers(rng, n_seq + 1, n, kind)), k, v, i32(numbers(rng, n_seq, m, "near")),
                              i32(numbers(rng, n_seq, m, "near")), o[:n], ws)
        torch.cuda.synchronize()
        assert (o[n:] == 7.0).all()


@pytest.mark.parametrize("kind", ["any", "near", "turns"])
@pytest.mark.parametrize("n_seq,n", [(2, 400), (64, 200), (65, 3000), (500, 300)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_the_cache(e4m3, n_seq, n, kind):
    rng = np.random.default_rng(n_seq + 1)
    n_pages, max_pages = 50, 40
    p = B.make_cache_params(n_seq, 4, 64, kv_heads=2, cache_dtype=int(e4m3), page_tokens=16, n_pages=n_pages + 2, max_pages=max_pages, frame_tokens=1)
    c = B.alloc_cache(p)
    p.n_pages = n_pages                                    # (the pool's last two pages are nobody's)
    c.page_table.copy_(i32(np.where(rng.random((n_seq, max_pages)) < 0.1, rng.integers(-2 ** 31, 2 ** 31, (n_seq, max_pages)),
                                    rng.integers(-1, n_pages + 3, (n_seq, max_pages)))))
    pools = [x for x in (c.k, c.v, c.k_scale, c.v_scale) if x is not None]
    for x in pools:
        x.fill_(56)
    k, v = randn(n, 2, 64), randn(n, 2, 64)
    off, pos = i32(numbers(rng, n_seq + 1, n, kind)), i32(numbers(rng, n_seq, 16 * max_pages, kind))
    B.litevggt_cache_write(p, c, k, v, off, pos)
    torch.cuda.synchronize()
    assert all((x[n_pages:] == 56).all() for x in pools)
    out = [torch.full((n + BEHIND, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.litevggt_cache_read(p, c, pos, off, out[0][:n], out[1][:n])
    o = torch.full((n + BEHIND, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.litevggt_cached_attn(p, c, randn(n, 4, 64), off, pos, o[:n], B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n)).fill_(255))
    torch.cuda.synchronize()
    assert all((x[n:] == 7.0).all() for x in (*out, o))


def test_sums_beyond_32_bits():
    """Every other one of 60,000 sequences claims all of 100,000 rows of 64 heads: 6e9 blocks of 32 rows, where the room is 4e6."""
    n_seq, heads, n = 60000, 64, 100000
    q, k = randn(n, heads, 64), randn(64, heads, 64)
    o = torch.full((n + BEHIND, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    p = B.make_cross_params(n_seq, heads, 64)
    ws = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(p, n, 64)).fill_(255)
    B.litevggt_cross_attn(p, q, i32(np.arange(n_seq + 1) % 2 * n), k, k, i32([0] * n_seq), i32([64] * n_seq), o[:n], ws)
    torch.cuda.synchronize()
    assert (o[n:] == 7.0).all()
    # the first sequence's claim comes first, and whole (each side off by 2^-8 of the result and of sum w |v| / sum w, both at most max |v|)
    part = torch.full((40, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    one = B.make_cross_params(1, heads, 64)
    B.litevggt_cross_attn(one, q[:40], i32([0, 40]), k, k, i32([0]), i32([64]), part, B.alloc_ws(B.litevggt_cross_attn_ws_bytes(one, 40, 64)))
    assert (o[:40].float() - part.float()).abs().max() <= 2.0 ** -6 * k.abs().max().item()
