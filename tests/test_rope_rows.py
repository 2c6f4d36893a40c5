"""Which rows the outputs of a rotation may lie in: host code, no GPU.  A call whose rows are in order gets as far as the launch, which needs a
device; it is told from a refusal by its code."""
import ctypes as C

import pytest

from paper_2512_04939_amd import binding as B

SHAPE = -2
P = 1 << 30      # stands for a device pointer
HEADS, KV, DIM, N = 4, 2, 64, 5
W, KW = HEADS * DIM, KV * DIM


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    """Without a device nothing is launched; with one these calls may not be made."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("pointers of no memory")


def rope(q, qs, k, ks, qo, qos, ko, kos, n=N, kv=KV):
    p = B.make_rope_params(HEADS, DIM, (16, 16), kv_heads=kv)
    at = lambda x: P + 2 * x      # noqa: E731
    return B.lib().litevggt_rope(C.byref(p), n, P + (1 << 28), at(q), qs, at(k), ks, at(qo), qos, at(ko), kos, None)


FAR = 1 << 20      # elements: another tensor


@pytest.mark.parametrize("q,qs,k,ks,qo,qos,ko,kos", [
    (0, W, FAR, KW, 0, W + 8, 2 * FAR, KW),                        # q's output in q's place, rows another way apart
    (0, 2 * W, FAR, KW, 0, W, 2 * FAR, KW),
    (0, W, FAR, KW, 2 * FAR, W, FAR, KW + 8),                      # k's
    (0, W, FAR, KW, 8, W, 2 * FAR, KW),                            # a few channels on
    (8, W, FAR, KW, 0, W, 2 * FAR, KW),
    (0, W, FAR, KW, W, W, 2 * FAR, KW),                            # a row on
    (0, W, FAR, KW, (N - 1) * W, W, 2 * FAR, KW),                  # its first row is q's last
    (0, W, FAR, KW, FAR, W, 2 * FAR, KW),                          # q's output in k's place
    (0, W, FAR, KW, 2 * FAR, W, 0, KW),                            # k's in q's
    (0, W, FAR, KW, 2 * FAR, W, 2 * FAR, KW),                      # both in one
    (0, W + KW, W, W + KW, FAR, W + KW, FAR + W - 8, W + KW),      # slices that meet
    (0, W, FAR, KW, FAR + 3 * W, 5 * W, FAR + 3 * W + 2 * KW, 2 * KW),
], ids=str)
def test_outputs_that_meet_other_rows_are_refused(q, qs, k, ks, qo, qos, ko, kos):
    assert rope(q, qs, k, ks, qo, qos, ko, kos) == SHAPE


@pytest.mark.parametrize("q,qs,k,ks,qo,qos,ko,kos,n", [
    (0, W, FAR, KW, 2 * FAR, W, 3 * FAR, KW, N),
    (0, W, FAR, KW, 0, W, FAR, KW, N),                             # in place
    (0, W + KW, W, W + KW, 0, W + KW, W, W + KW, N),               # in place, slices of one projection's output
    (0, 3 * W, W, 3 * W, FAR, W + KW, FAR + W, W + KW, N),         # out of one, into another
    (0, 3 * W, W, 3 * W, 2 * W, 3 * W, FAR, KW, N),                # q's output between the slices
    (0, W, FAR, KW, N * W, W, FAR + N * KW, KW, N),                # behind each other
    (N * W, W, FAR, KW, 0, W, 2 * FAR, KW, N),
    (0, W, 0, W, FAR, W, 2 * FAR, KW, N),                          # inputs may meet
    (0, W, FAR, KW, 0, W + 8, FAR, 4 * KW, 1),                     # one row has no stride
    (0, W, FAR, KW, FAR + 3 * W, 5 * W, FAR + 4 * W, 5 * W, N),
    (0, 4 * W, FAR, KW, W, 8 * W, 2 * FAR, KW, N),                 # rows of unlike strides side by side
], ids=str)
def test_other_rows_are_not(q, qs, k, ks, qo, qos, ko, kos, n):
    assert rope(q, qs, k, ks, qo, qos, ko, kos, n) != SHAPE


def test_without_k_its_rows_are_not_looked_at():
    assert rope(0, W, 0, KW, FAR, W, 0, KW + 8, kv=0) != SHAPE
    assert rope(0, W, FAR, KW, 0, W + 8, FAR, KW, kv=0) == SHAPE
