"""Attention over an E2M1 cache where a wave walks its list of pages further than the 64 tiles (few rows) or stages (many) that it looks up at a
time, against the definition in 64 bits.  Pages of a small pool stand in many columns.

Tolerance as in stream_cases.Pool.attend: a weight and the result rounded to bf16, 2^-8 each; a score's error is a weight's, twice with its row's
sum and doubled for the exponential's own."""
import numpy as np
import pytest
import torch

from paper_2512_04939_amd import binding as B

from stream_cases import Pool, dev, i32, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("n_seq,kv,group,dim,new,length", [
    (16, 128, 1, 64, 1, 20000),      # 2048 units of 157 tiles in three rounds of 1024 places: 104 tiles to a piece
    (16, 64, 2, 128, 1, 20000),      # 1024 units, three rounds of 512 places
    (16, 64, 1, 64, 40, 17000),      # rows in blocks of 64
    (130, 16, 1, 64, 65, 9000),      # many rows, not cut: 141 stages
    (130, 16, 1, 128, 40, 9000),
], ids=str)
def test_long_lists(n_seq, kv, group, dim, new, length, page):
    c = Pool(71, [18 * page], heads=kv * group, kv_heads=kv, head_dim=dim, page=page, spare=0)
    rng = c.rng
    lens = [length] + [int(x) for x in rng.integers(length // 2, length + 1, n_seq - 1)]
    columns = -(-length // page)
    t = np.full((n_seq, columns), -1, np.int32)
    for s, n in enumerate(lens):
        used = -(-n // page)
        t[s, :used] = np.where(rng.random(used) < 0.1, -1, rng.integers(0, c.n_pages, used))
    t[0, 8192 // page:8704 // page] = -1        # a run behind the first look-up of the longest
    p = B.make_cache_params(n_seq, kv * group, dim, kv_heads=kv, cache_dtype=B.CACHE_E2M1, page_tokens=page, n_pages=c.n_pages, max_pages=columns,
                            frame_tokens=3)
    c.d.page_table = torch.from_numpy(t).cuda()
    q = dev(rows(rng, n_seq * new, kv * group, dim))
    o = torch.full_like(q, float("nan"))
    ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n_seq * new)).fill_(255)
    B.litevggt_cached_attn(p, c.d, q, i32(new * s for s in range(n_seq + 1)), i32(lens), o, ws)
    assert torch.isfinite(o).all()
    k_all, v_all = torch.from_numpy(c.o.k).cuda(), torch.from_numpy(c.o.v).cuda()
    norm = float(q.double().square().sum(-1).max().sqrt()) * float(k_all.square().sum(-1).max().sqrt())
    error = dim ** -0.5 * dim * 2.0 ** -24 * norm
    for s in sorted({0, 1, n_seq // 2, n_seq - 1}):
        at = torch.arange(lens[s], device="cuda")
        ids = c.d.page_table[s].long()[at // page]
        k, v = k_all[ids.clamp(min=0), :, at % page], v_all[ids.clamp(min=0), :, at % page]
        pos = torch.arange(lens[s] - new, lens[s], device="cuda")
        seen = (ids >= 0) & (at < ((pos // 3 + 1) * 3)[:, None])
        for h in {0, 1, kv * group // 2, kv * group - 1}:
            z = (q[s * new:(s + 1) * new, h].double() @ k[:, h // group].t().contiguous() * dim ** -0.5).masked_fill(~seen, -torch.inf)
            w, x = torch.softmax(z, 1), v[:, h // group].contiguous()
            exact, spread = w @ x, w @ x.abs()
            off = (o[s * new:(s + 1) * new, h].double() - exact).abs()
            assert bool((off <= 2.0 ** -8 * exact.abs() + (2.0 ** -8 + 4 * error) * spread).all()), (s, h, float(off.max()))
