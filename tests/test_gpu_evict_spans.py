"""Eviction on the GPU where a workgroup sums several spans of a sequence, one after the other (exact, as in test_gpu_evict)."""
import numpy as np
import pytest

from test_gpu_evict import run, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads,n_seq,longest", [
    (16, 1, 32, 80000),          # 313 spans of 256 positions on 256 workgroups
    (64, 5, 32, 70001), (256, 1, 40, 105000), (1024, 2, 64, 100000),
    (16, 1, 9000, 700),          # one workgroup to a sequence, up to three spans
])
def test_spans_in_turns(page, heads, n_seq, longest):
    rng = np.random.default_rng(page + n_seq)
    lens = [longest] + [int(x) for x in rng.integers(0, longest + 1, n_seq - 1)]
    spans = -(-(-(-longest // page) * page) // 256)
    assert spans * n_seq > 8192 and spans > max(1, 8192 // n_seq)
    pages = [-(-n // page) for n in lens]
    columns, n_pages = max(pages) + 1, sum(pages) + 2
    t = tables(rng, pages, columns, n_pages)
    mass = (rng.random((n_seq, heads, columns * page), dtype=np.float32) ** 2)
    mass *= (rng.random((n_seq, 1, columns)) < 0.8).repeat(page, 2)          # pages that drew nothing: ties
    run(t, n_pages, page, lens, mass, [c // 2 for c in pages], 1, 1)
