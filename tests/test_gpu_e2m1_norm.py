"""Queries that the call normalises: attention over an E2M1 cache, and the drawn weight over every type, in the forms of few and of many rows;
attention over an E2M1 cache gives the same bits again.

Half of a query's channels are +-2^j and half +-2^(j + 1): its root mean square is 2^j sqrt(2.5) and the normalised values are 0.6325 and
1.2649, four tenths of a bf16 step from where their rounding changes, which 32 bits cannot reach.  So a score is off by its sums alone."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2512_04939_amd import binding as B

from stream_cases import DTYPES, Pool, dev, i32, rows

pytestmark = pytest.mark.gpu


class Normed(Pool):
    def __init__(self, seed, lens, **kw):
        super().__init__(seed, lens, qk_norm=1, **kw)

    def queries(self, n):
        d = self.p.head_dim
        size = np.repeat([1.0, 2.0], d // 2)
        q = np.empty((n, self.p.heads, d))
        for row in q.reshape(-1, d):
            row[:] = self.rng.permutation(size) * self.rng.choice([-1.0, 1.0], d) * 2.0 ** self.rng.integers(0, 12)
        z = O.normed(q)
        assert set(np.unique(np.abs(z))) == {O.round_bf16(0.4 ** 0.5).item(), O.round_bf16(1.6 ** 0.5).item()}
        return q

    def score_error(self, q):
        """stream_cases.Pool's without values that fall to the other side of a border."""
        k = np.sqrt((self.o.k ** 2).sum(-1)).max()
        return self.softmax_scale() * self.p.head_dim * 2.0 ** -24 * np.sqrt((O.normed(q) ** 2).sum(-1)).max() * k


SIZES = [
    # one row; some; more than 32 (two blocks of 32 at 64 channels); many; cut into pieces; unlike sequences
    dict(lens=[90], new=[1], heads=2), dict(lens=[301, 40], new=[3, 1], heads=8, kv_heads=2, frame=1), dict(lens=[500], new=[50], heads=2, frame=20),
    dict(lens=[700], new=[300], heads=2, page=32, frame=1), dict(lens=[2600], new=[7], heads=2), dict(lens=[333, 90, 0], new=[150, 1, 0], heads=4, kv_heads=2),
]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_attention_over_e2m1(size, dim):
    size = dict(size)
    lens, new = size.pop("lens"), size.pop("new")
    size.setdefault("kv_heads", size["heads"])
    c = Normed(61, lens, head_dim=dim, holes=[(0, 2)], **size)
    c.attend(new, q=c.queries(sum(new)))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_drawn_weight(size, dim, dtype):
    size = dict(size)
    lens, new = size.pop("lens"), size.pop("new")
    size.setdefault("kv_heads", size["heads"])
    c = Normed(62, lens, head_dim=dim, dtype=dtype, holes=[(0, 2)], **size)
    c.draw(new, q=c.queries(sum(new)))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("norm", [0, 1])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_attention_over_e2m1_gives_the_same_bits_again(new, norm, dim):
    """With scratch of any contents, and that of a longer call."""
    c = Pool(63, [3000, 700], heads=4, kv_heads=2, head_dim=dim, qk_norm=norm, frame=1, holes=[(0, 5), (1, 30)])
    p, off, length = c.p, i32([0, new, 2 * new]), i32(c.lens)
    q = dev(rows(c.rng, 2 * new, 4, dim))
    outs = []
    for fill, n in ((255, 2 * new), (0, 2 * new), (127, 2 * new), (255, 5000)):
        ws = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, n)).fill_(fill)
        o = torch.full_like(q, float("nan"))
        B.litevggt_cached_attn(p, c.d, q, off, length, o, ws)
        outs.append(o)
    assert all(torch.equal(outs[0], o) for o in outs[1:])
