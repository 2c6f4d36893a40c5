"""Pins of the plain implementation of the paged cache and of attention over it against independent formulations."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as O


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal(20000) * 10.0 ** np.random.default_rng(1).uniform(-30, 30, 20000)
    x[:4] = [1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -(1 + 2.0 ** -8), 0.0]       # ties
    f = x.astype(np.float32)
    assert np.array_equal(O.round_bf16(f.astype(np.float64)), torch.from_numpy(f).bfloat16().double().numpy())
    assert O.round_bf16(1 + 2.0 ** -8 + 2.0 ** -40) == 1 + 2.0 ** -7         # what float32 would make a tie


def test_e4m3_values_and_rounding_are_torchs():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_values(), codes, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 40001), np.random.default_rng(2).standard_normal(20000) * 0.02])
    f = x.astype(np.float32)
    assert np.array_equal(O.round_e4m3(f.astype(np.float64)), torch.from_numpy(f).to(torch.float8_e4m3fn).double().numpy())
    assert O.round_e4m3(np.array([1e9, -1e9, np.inf])).tolist() == [448.0, -448.0, 448.0]


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, 0), (2.0 ** -133, -126), (3.3e38, 120)])
def test_row_exponent(top, e):
    row = np.array([0.0, -top, top / 3, np.inf, np.nan])
    assert O.row_exponent(row) == e
    if top > 0 and e > -126:
        assert top <= 448 * 2.0 ** e and top > 448 * 2.0 ** (e - 1)


def test_attention_against_torch():
    g = torch.Generator().manual_seed(0)
    q = torch.randn(9, 6, 64, generator=g, dtype=torch.float64)
    k, v = (torch.randn(33, 2, 64, generator=g, dtype=torch.float64) for _ in range(2))
    seen = torch.rand(9, 33, generator=g) < 0.5
    seen[4] = False
    ref = torch.nn.functional.scaled_dot_product_attention(
        q.transpose(0, 1), k.repeat_interleave(3, 1).transpose(0, 1), v.repeat_interleave(3, 1).transpose(0, 1),
        attn_mask=seen).transpose(0, 1)
    got = O.attend(q.numpy(), k.numpy(), v.numpy(), seen.numpy(), 1 / 8)
    assert np.all(got[4] == 0)
    live = [i for i in range(9) if i != 4]
    np.testing.assert_allclose(got[live], ref.numpy()[live], rtol=1e-12, atol=1e-12)


def test_what_a_row_does_not_see_has_no_part_in_it():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((4, 2, 64)), rng.standard_normal((8, 2, 64)), rng.standard_normal((8, 2, 64))
    seen = np.tril(np.ones((4, 8), bool), 1)
    clean = O.attend(q, k, v, seen, 1.0)
    k[5], v[5, 0, 3], v[4, 1, 7], v[2, 1, 9] = np.nan, np.inf, np.nan, np.inf
    got = O.attend(q, k, v, seen, 1.0)
    assert np.isinf(got[1:, 1, 9]).all() and np.isnan(got[3:, 1, 7]).all()
    got[1:, 1, 9], got[3:, 1, 7] = clean[1:, 1, 9], clean[3:, 1, 7]
    np.testing.assert_array_equal(got, clean)


def test_frames_one_after_another_are_frame_causal_attention_over_all():
    """Six frames of five tokens through the cache, a frame per call, against one call over the whole sequence with
    a mask, and a frame's row against a loop over its keys."""
    rng = np.random.default_rng(4)
    T, F, heads, kv, d = 5, 6, 4, 2, 64
    n = T * F
    q = rng.standard_normal((n, heads, d))
    k, v = rng.standard_normal((n, kv, d)), rng.standard_normal((n, kv, d))
    table = np.array([[3, 0, 4]])
    cache = O.Cache(5, kv, 16, d, table, False)
    out = []
    for f in range(F):
        cache.write(k[f * T:(f + 1) * T], v[f * T:(f + 1) * T], [0, T], [f * T])
        out.append(O.cached_attention(cache, q[f * T:(f + 1) * T], [0, T], [(f + 1) * T], T))
    frame = np.arange(n) // T
    ref = O.attend(q, k, v, frame[:, None] >= frame[None, :], 1 / 8)
    np.testing.assert_allclose(np.concatenate(out), ref, rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(O.cached_attention(cache, q, [0, n], [n], T), ref, rtol=1e-12, atol=1e-14)
    w = [math.exp(float(q[7, 3] @ k[t, 1]) / 8) for t in range(10)]
    np.testing.assert_allclose(ref[7, 3], sum(a * v[t, 1] for t, a in enumerate(w)) / sum(w), rtol=1e-12)


def test_cache_round_trip_and_pages_that_are_not_held():
    rng = np.random.default_rng(5)
    k, v = (O.round_bf16(rng.standard_normal((40, 2, 64)) * 5) for _ in range(2))
    table = np.array([[2, -1, 0], [9, 1, -1]])
    for e4m3 in (False, True):
        cache = O.Cache(3, 2, 16, 64, table, e4m3)
        cache.write(k, v, [0, 30, 40], [5, 20])
        rk, rv, held = cache.rows(0, 0, 40)
        assert held.tolist() == [i // 16 != 1 for i in range(40)]
        assert np.all(rk[:5] == 0) and np.all(rk[16:32] == 0)
        tol = 0 if not e4m3 else 2.0 ** -4
        assert np.all(np.abs(rk[5:16] - k[:11]) <= tol * np.abs(k[:11]) + tol * 2.0 ** -6 * 16)
        assert np.all(np.abs(cache.rows(1, 20, 10)[1] - v[30:]) <= tol * np.abs(v[30:]) + tol * 2.0 ** -6 * 16)
        assert not cache.rows(1, 0, 16)[2].any()       # a page number beyond the pool


def test_cross_attention_ranges():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((7, 2, 64)), rng.standard_normal((20, 1, 64)), rng.standard_normal((20, 1, 64))
    got = O.cross_attention(q, [1, 3, 3, 6], k, v, [0, 4, 10], [20, 9, 10])
    assert np.isnan(got[[0, 6]]).all() and np.all(got[3:6] == 0)
    np.testing.assert_allclose(got[1:3], O.attend(q[1:3], k, v, np.ones((2, 20), bool), 1 / 8))
