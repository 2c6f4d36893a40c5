"""Pins of the plain implementation of rotary positions, the E2M1 cache, drawn weight and eviction against brute force and invariants."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as O
from oracle import stream_oracle as S


def test_e2m1_codes_are_the_nearest_and_ties_go_to_even():
    values = [S.e2m1_value(c) for c in range(8)]
    assert values == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    for a, b, want in ((0, 0.5, 0.0), (0.5, 1, 1.0), (1, 1.5, 1.0), (1.5, 2, 2.0), (2, 3, 2.0), (3, 4, 4.0), (4, 6, 4.0)):
        mid = (a + b) / 2
        assert S.e2m1_value(S.e2m1_code(mid)) == want and S.e2m1_value(S.e2m1_code(-mid)) == -want
        assert S.e2m1_value(S.e2m1_code(mid - 1e-9)) == a and S.e2m1_value(S.e2m1_code(mid + 1e-9)) == b
    assert S.e2m1_code(-0.0) == 8 and S.e2m1_code(0.0) == 0


def test_block_exponent():
    one = lambda v: S.block_exponent(np.array([v] + [0.0] * 31))     # noqa: E731
    assert one(6.0) == 0 and one(6.0000001) == 1 and one(3.0) == -1 and one(0.0) == 0 and one(2.0 ** -140) == -126
    assert one(math.inf) == 0 and one(math.nan) is None
    x, e, c = S.round_blocks(np.array([[12.0, -math.inf, 1.0] + [0.0] * 29 + [math.nan] * 1 + [1.0] * 31]))
    assert e.tolist() == [[1, 128]] and x[0, :3].tolist() == [12.0, -12.0, 1.0] and np.isnan(x[0, 32:]).all()


def test_weights_drawn_add_up_to_the_rows_that_see_something():
    rng = np.random.default_rng(0)
    table = np.array([[0, -1, 2, 3], [-1, -1, -1, -1]])
    c = O.Cache(4, 2, 16, 64, table, False)
    c.k = rng.standard_normal(c.k.shape)
    q = rng.standard_normal((5, 4, 64))
    had = rng.random((2, 2, 64))
    out = S.mass(c, q, [0, 3, 5], [50, 9], 7, had, np.full((2, 2, 64), 5.0))
    held = np.repeat(table >= 0, 16, 1)
    drawn = (out - had)[0, :, :50][:, held[0, :50]]
    assert np.allclose(drawn.sum(1), 3 * 2)
    assert (out[0, :, 16:32] == 0).all() and (out[0, :, 50:] == 5).all() and (out[1, :, :9] == 0).all() and (out[1, :, 9:] == 5).all()


def test_evict_keeps_what_it_should():
    table = np.array([[5, -1, 3, 9, 0, 7]])
    mass = np.repeat(np.array([[1.0, 0.0, 0.25, 0.25, 9.0, 0.0]]), 16, 1)[None]
    out, freed, n = S.evict(table, 10, 16, [96], mass, [3], 0, 0)
    assert out.tolist() == [[5, -1, -1, 9, 0, -1]] and freed.tolist() == [[3, 7, -1, -1, -1, -1]] and n.tolist() == [2]
    out, freed, n = S.evict(table, 10, 16, [90], mass, [0], 1, 2)
    assert out.tolist() == [[5, -1, -1, -1, 0, 7]] and n.tolist() == [2]
    out, _, n = S.evict(table, 4, 16, [96], mass, [0], 0, 0)              # 5, 9 and 7 are no pages of a pool of 4
    assert out.tolist() == [[5, -1, -1, 9, -1, 7]] and n.tolist() == [2]


@pytest.mark.parametrize("pairing", [0, 1, 2])
@pytest.mark.parametrize("joint", [False, True])
def test_rotation_keeps_lengths_and_scores_by_distance(pairing, joint):
    rng = np.random.default_rng(1)
    pairs = (5, 9, 11)
    q, k = rng.standard_normal((2, 1, 1, 64))
    turn = lambda x, p, inv=False: S.rope(x, np.array([p]), pairs, pairing, joint, inv, base=100.0)     # noqa: E731
    a = turn(q, (3, 10, 4))
    assert np.allclose((a ** 2).sum(), (q ** 2).sum()) and np.allclose(turn(a, (3, 10, 4), True), q)
    assert np.array_equal(a[..., 50:], q[..., 50:]) and np.array_equal(turn(q, (0, 0, 0)), q)
    one = (turn(q, (3, 10, 4)) * turn(k, (1, 2, 3))).sum()
    assert np.allclose(one, (turn(q, (13, 30, 104)) * turn(k, (11, 22, 103))).sum())
