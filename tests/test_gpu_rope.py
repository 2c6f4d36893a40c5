"""Rotary positions on the GPU against the plain implementation in 64 bits.

Tolerance: the result is rounded to bf16 (2^-8 of it); the angle's fraction of a turn is a 32-bit number (off by 2^-25 turns, and by 2^-24 more
at the largest positions), the sine and cosine are the hardware's, taken as good to 2^-16, so y is off by 2^-15 (|x1| + |x2|) beside."""
import numpy as np
import pytest
import torch

from oracle import stream_oracle as S
from paper_2512_04939_amd import binding as B

from stream_cases import dev, host, i32, rows

pytestmark = pytest.mark.gpu


def check(got, x, exact):
    size = np.abs(x).max(-1, keepdims=True) * 2
    assert not (np.abs(got - exact) > 2.0 ** -8 * np.abs(exact) + 2.0 ** -15 * size).any(), np.abs(got - exact).max()


def case(seed, n, heads, kv, dim, pairs, pairing, joint, inverse, far, base=100.0, freq=None):
    rng = np.random.default_rng(seed)
    p = B.make_rope_params(heads, dim, pairs, kv_heads=kv, pairing=pairing, joint=joint, inverse=inverse, base=base, freq=freq)
    q, k = rows(rng, n, heads, dim), rows(rng, n, kv, dim)
    pos = rng.integers(-far, far + 1, (n, len(pairs))).astype(np.int32)
    return p, q, k, pos


SHAPES = [(1, 16, 16, 64, (16, 16)), (5, 4, 1, 64, (32,)), (33, 3, 2, 64, (8, 12, 12)), (70, 8, 2, 128, (16, 24, 24)), (17, 1, 0, 128, (5, 7, 1, 3)),
          (2, 17, 5, 64, (1,)), (257, 2, 2, 128, (64,)), (3, 40, 8, 128, (8, 8, 8, 8))]


@pytest.mark.parametrize("pairing", [B.ROPE_AXIS_HALVES, B.ROPE_HEAD_HALVES, B.ROPE_ADJACENT])
@pytest.mark.parametrize("joint,inverse", [(0, 0), (1, 1)])
@pytest.mark.parametrize("n,heads,kv,dim,pairs", SHAPES, ids=str)
def test_rotation(n, heads, kv, dim, pairs, pairing, joint, inverse):
    p, q, k, pos = case(1, n, heads, kv, dim, pairs, pairing, joint, inverse, 1000)
    q[0, 0, -1] = -0.0
    qd, kd = dev(q), dev(k)
    qo, ko = torch.full_like(qd, 7.0), torch.full_like(kd, 7.0)
    pd = torch.from_numpy(pos).cuda()
    B.litevggt_rope(p, pd, qd, kd if kv else None, qo, ko if kv else None)
    for x, y in ((q, qo), (k, ko)):
        if x.size:
            check(host(y), x, S.rope(x, pos, pairs, pairing, joint, inverse, base=p.base))
            if 2 * sum(pairs) < dim:
                assert np.array_equal(host(y)[..., 2 * sum(pairs):], x[..., 2 * sum(pairs):])
    # in place, and as slices of one projection's output
    both = torch.cat([qd.flatten(1), kd.flatten(1)], 1)
    qs, ks = both[:, :heads * dim].unflatten(1, (heads, dim)), both[:, heads * dim:].unflatten(1, (kv, dim)) if kv else None
    B.litevggt_rope(p, pd, qs, ks, qs, ks)
    assert torch.equal(qs, qo) and (not kv or torch.equal(ks, ko))


@pytest.mark.parametrize("far", [2 ** 31 - 1, 2 ** 24 + 1, 3])
@pytest.mark.parametrize("base", [100.0, 500000.0, 1.0])
def test_far_positions(far, base):
    p, q, k, pos = case(2, 41, 2, 2, 64, (8, 24), B.ROPE_AXIS_HALVES, 0, 0, far, base=base)
    pos[0], pos[1] = far, -far
    qo, ko = dev(q), dev(k)
    B.litevggt_rope(p, torch.from_numpy(pos).cuda(), qo, ko, qo, ko)
    # 64 bits hold position times frequency to 2^-22 at 2^31, which the oracle's remainder of 2 pi inherits: another 2^-20
    for x, y in ((q, qo), (k, ko)):
        exact = S.rope(x, pos, (8, 24), 0, False, False, base=base)
        assert not (np.abs(host(y) - exact) > 2.0 ** -8 * np.abs(exact) + 2.0 ** -14 * np.abs(x).max(-1, keepdims=True)).any()


def test_frequencies_of_its_own():
    freq = [0.5, -1.25, 3.0, 0.0, 100.0]
    p, q, k, pos = case(3, 20, 2, 1, 64, (2, 3), B.ROPE_ADJACENT, 0, 0, 50, freq=freq)
    qo, ko = dev(q), dev(k)
    B.litevggt_rope(p, torch.from_numpy(pos).cuda(), qo, ko, qo, ko)
    check(host(qo), q, S.rope(q, pos, (2, 3), 2, False, False, freq=freq))
    check(host(ko), k, S.rope(k, pos, (2, 3), 2, False, False, freq=freq))


@pytest.mark.parametrize("pairing", [0, 1, 2])
def test_inverse_is_the_gradient(pairing):
    """<rope(x), g> = <x, inverse(g)>, for the formula and for differences of the forward pass."""
    pairs = (16, 24, 24)
    p, q, _, pos = case(4, 9, 3, 0, 128, pairs, pairing, 1, 0, 300)
    back = B.make_rope_params(3, 128, pairs, kv_heads=0, pairing=pairing, joint=1, inverse=1)
    rng = np.random.default_rng(5)
    g, pd = rows(rng, 9, 3, 128), torch.from_numpy(pos).cuda()
    dx = torch.empty(9, 3, 128, dtype=torch.bfloat16, device="cuda")
    B.litevggt_rope(back, pd, dev(g), None, dx, None)
    check(host(dx), g, S.rope(g, pos, pairs, pairing, True, True, base=100.0))
    # differences: the rotation is linear, so a step of any size does; both sides are rounded
    step = np.zeros_like(q)
    step[4, 1, 37] = 8.0
    y = [torch.empty_like(dx) for _ in range(2)]
    for out, x in zip(y, (np.zeros_like(q), step)):
        B.litevggt_rope(p, pd, dev(x), None, out, None)
    change = ((host(y[1]) - host(y[0])) / 8.0 * g).sum()
    assert abs(change - host(dx)[4, 1, 37]) <= (2.0 ** -8 + 2.0 ** -14) * 4 * np.abs(g[4, 1]).max()


def test_what_is_not_finite_stays_in_its_pair():
    p = B.make_rope_params(1, 64, (8, 8), kv_heads=0)
    x = np.ones((2, 1, 64))
    x[0, 0, 3], x[1, 0, 50] = np.nan, np.inf
    y = dev(x)
    B.litevggt_rope(p, torch.ones(2, 2, dtype=torch.int32, device="cuda"), y, None, y, None)
    got = host(y)
    assert np.isnan(got[0, 0, [3, 11]]).all() and np.isfinite(np.delete(got[0, 0], [3, 11])).all()
    assert got[1, 0, 50] == np.inf and np.isfinite(np.delete(got[1, 0], 50)).all()


def test_no_tokens_and_a_replayed_graph():
    p = B.make_rope_params(2, 64, (16, 16))
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.litevggt_rope(p, torch.empty(0, 2, dtype=torch.int32, device="cuda"), none, none, none, none)
    rng = np.random.default_rng(6)
    q, pos = dev(rows(rng, 7, 2, 64)), torch.ones(7, 2, dtype=torch.int32, device="cuda")
    out = [torch.empty_like(q) for _ in range(2)]
    B.litevggt_rope(p, pos, q, q, *out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.litevggt_rope(p, pos, q, q, *out)
    for t in (3, 77, 12345):
        pos.fill_(t)
        g.replay()
        torch.cuda.synchronize()
        again = [torch.empty_like(q) for _ in range(2)]
        B.litevggt_rope(p, pos, q, q, *again)
        assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1]) and torch.equal(out[0], out[1])
