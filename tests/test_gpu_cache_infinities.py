"""Infinities and NaN of V in positions that queries do see: the result has the class and the sign that the sum has in 64 bits, wherever
the key falls in the tiling.  Tolerances of the finite entries as in test_gpu_cache (roundings of weights and result)."""
import numpy as np
import pytest

from test_gpu_cache import Case, rows, run_cross

pytestmark = pytest.mark.gpu


def same(got, exact, tol):
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(kind(got), kind(exact)), (kind.__name__, np.argwhere(kind(got) != kind(exact))[:5])
    fine = np.isfinite(exact)
    assert np.all(np.abs(got[fine] - exact[fine]) <= tol[fine])


def wild(v, first, last):
    """V's rows by position [position][kv head][channel] get entries that are not finite: the first, the last and one between."""
    v[first][0, 3] = v[first][-1, 40] = np.inf
    v[last][0, 7] = -np.inf
    v[first][0, 11], v[last][0, 11] = np.inf, -np.inf          # NaN for those who see both
    v[(first + last) // 2][0, 50] = np.nan
    v[(first + last) // 2][-1, 60] = -np.inf


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,new,frame", [
    # one key to a few, less than a tile, a prompt (all positions new), the diagonal of longer ones, the ragged end of cut ones
    ([1], [1], 1), ([2], [2], 1), ([5, 20], [5, 3], 1), ([20], [20], 1), ([31], [1], 0), ([40], [40], 7), ([100], [100], 1),
    ([127], [33], 0), ([300], [300], 1), ([300, 90], [300, 90], 50), ([9001], [5], 0), ([9001], [40], 1), ([9001], [200], 1),
])
def test_cached_attention_of_infinite_values(lens, new, frame, dim):
    c = Case(41, lens, heads=4, kv_heads=2, head_dim=dim, page=16, frame=frame)
    for s, n in enumerate(lens):
        at = [c.o.place(s, t) for t in range(n)]
        wild([c.o.v[page, :, row] for page, row in at], 0, n - 1)
    c.d = c.device()
    same(*c.attend(new))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,ranges", [([3], [(0, 1)]), ([5], [(2, 22)]), ([40, 2], [(0, 20), (7, 70)]), ([150], [(1, 41)]), ([90, 200], [(0, 33), (3, 300)])])
def test_cross_attention_of_infinite_values(nq, ranges, dim):
    rng = np.random.default_rng(42)
    v = rows(rng, 300, 2, dim)
    for first, last in ranges:
        wild(v, first, last - 1)
    same(*run_cross(rng, nq, ranges, 300, 4, 2, dim, v=v))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 40, 200])
def test_an_infinity_at_a_key_of_far_the_largest_score(new, dim):
    """The key that raises a row's reference by hundreds of binades is the one whose value is infinite."""
    c = Case(43, [70 + new], heads=2, kv_heads=1, head_dim=dim, page=16, frame=0)
    for t in range(70 + new):
        page, row = c.o.place(0, t)
        c.o.k[page, 0, row] = 8.0 if t == 68 + new else 0.0
        c.o.v[page, 0, row, 5] = -np.inf if t == 68 + new else 1.0
    c.d = c.device()
    # (scores 8 * 10 * dim / sqrt(dim) = 640 or 905 against 0, products and sums exact)
    same(*c.attend([new], q=np.full((new, 2, dim), 10.0)))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [2, 40, 200])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_as_large_as_allowed(sign, new, dim):
    """Scores of +-2^27 and half of that (64 channels; half as much again for 128): the keys of the larger ones share the weight, to the
    last bit (the next ones' is exp(-2^26))."""
    c = Case(44, [150 + new], heads=2, kv_heads=1, head_dim=dim, page=16, frame=0)
    for t in range(150 + new):
        page, row = c.o.place(0, t)
        c.o.k[page, 0, row] = sign * (2.0 ** 13 if t % 3 else 2.0 ** 12)
    c.d = c.device()
    got, exact, _ = c.attend([new], q=np.full((new, 2, dim), 2.0 ** 11))
    # equal weights, rounded equally: only the result's rounding is left, and fp32 sums of 300 values below 8
    assert np.all(np.abs(got - exact) <= 2.0 ** -8 * np.abs(exact) + 300 * 8 * 2.0 ** -24)
