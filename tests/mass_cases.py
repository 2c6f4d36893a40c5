"""Calls of the drawn weight that reach every kernel and every way in which keys are cut (``csrc/mass_plan.h``): what each is to select is
checked on the CPU, what it gives on the GPU.

Pages of a small pool stand in many columns of the table, so that long sequences cost little memory."""
from __future__ import annotations

import numpy as np
import torch

from stream_cases import DTYPES, S, Pool, dev, i32, rows
from paper_2512_04939_amd import binding as B

LEVEL = 32.0      # between two stairs: e^32 > 2^40, at which a sum raises its reference


def case(name, lens, new, *, heads=16, kv_heads=None, head_dim=64, page=16, room=0, frame=0, gone=(), dtypes=("bf16", "e4m3", "e2m1"),
         form, rows_chunks, keys_chunks, of=0, tokens=None):
    """`gone`: (sequence, first position, end) whose pages are not held.  `form` and the chunks of a piece (of sequence `of`): what is selected."""
    return dict(name=name, lens=lens, new=new, heads=heads, kv_heads=kv_heads or heads, head_dim=head_dim, page=page,
                columns=max([room] + lens) // page + 1, frame=frame, gone=list(gone), dtypes=dtypes, form=form, rows_chunks=rows_chunks,
                keys_chunks=keys_chunks, of=of, tokens=tokens)


def between(chunk, per, pieces):
    """Of a sequence's pieces of `per` chunks each: the first chunk of the first, a middle one of the second, the last one of the third and all
    of the fourth are not held, nor are some positions inside others."""
    at = [(0, 1), (per + per // 2, per + per // 2 + 1), (3 * per - 1, 3 * per), (3 * per, 4 * per)]
    assert pieces > 4
    return [(1, a * chunk, b * chunk) for a, b in at] + [(1, 4 * per * chunk + chunk // 2, 4 * per * chunk + chunk // 2 + 16)]


# a sequence that holds nothing, whose many rows and keys make its share of the work large: the pieces of the other are long
def beside(name, keys, queries, length, new, per_rows, per_keys, chunk, **kw):
    return case(name, [keys, length], [queries, new], gone=[(0, 0, keys)] + between(chunk, per_rows, -(-length // (chunk * per_rows))), of=1,
                rows_chunks=per_rows, keys_chunks=per_keys, **kw)


CASES = [
    # up to 32 rows, scores kept
    case("few_joined", [20000], [5], gone=[(0, 96, 128), (0, 4000, 4300), (0, 9000, 9016)], form="few 8 kept", rows_chunks=3, keys_chunks=1),
    case("few_own", [15990], [7], gone=[(0, 0, 64), (0, 8000, 8100)], frame=13, form="few 8 kept own", rows_chunks=2, keys_chunks=1),
    case("few_32_joined", [20000], [12], gone=[(0, 96, 128), (0, 4000, 4300)], form="few 32 kept", rows_chunks=3, keys_chunks=1),
    case("few_32_own", [15000], [11], frame=5, head_dim=128, form="few 32 kept own", rows_chunks=2, keys_chunks=1),
    case("few_added_in_turns", [67000], [1], heads=64, page=1024, form="few 8 kept", rows_chunks=33, keys_chunks=2),
    case("few_unlike", [9000, 300, 0, 7000], [3, 1, 1, 11], heads=32, kv_heads=16, head_dim=128, frame=4, dtypes=("bf16", "e4m3"),
         form="few 8 kept", rows_chunks=4, keys_chunks=1),
    # scores that would take more than their share of the workspace, and rows of 128 channels beyond those that are kept
    case("few_again", [20000], [8], page=1024, room=(1 << 20) + 1024, gone=[(0, 1024, 2048), (0, 9216, 10240)], form="few 8", rows_chunks=3, keys_chunks=2),
    case("few_again_128", [20000], [8], head_dim=128, page=1024, room=(1 << 20) + 1024, frame=3, dtypes=("bf16", "e2m1"), form="few 8", rows_chunks=3,
         keys_chunks=2),
    case("few_32_again", [19000], [31], head_dim=128, gone=[(0, 96, 128), (0, 4000, 4300)], frame=9, dtypes=("e4m3", "e2m1"), form="few 32",
         rows_chunks=3, keys_chunks=2),
    # many rows
    case("many", [1500], [90], room=12288, frame=50, gone=[(0, 130, 520)], form="many", rows_chunks=1, keys_chunks=1),
    case("many_128", [1500], [90], room=12288, head_dim=128, frame=1, gone=[(0, 130, 520)], form="many", rows_chunks=1, keys_chunks=1),
    case("many_whole", [1500], [96], room=12288, gone=[(0, 130, 520)], form="many", rows_chunks=1, keys_chunks=1),
    case("many_whole_128", [1400], [64], room=12288, head_dim=128, gone=[(0, 130, 520)], form="many", rows_chunks=1, keys_chunks=1),
    case("many_unlike", [700, 1, 0, 333], [100, 1, 5, 64], heads=8, kv_heads=4, room=12288, frame=7, form="many", rows_chunks=1, keys_chunks=1),
    beside("many_in_turns", 16384, 3000, 5000, 30, 3, 6, 256, form="many"),
    beside("many_in_turns_frames", 16384, 3000, 5000, 60, 2, 3, 256, frame=17, form="many"),
    beside("many_in_turns_whole", 16384, 3000, 5000, 64, 2, 3, 256, form="many"),
    beside("many_in_turns_128", 16384, 3000, 4010, 30, 6, 12, 128, head_dim=128, frame=11, form="many"),
    beside("many_in_turns_128_whole", 16384, 3000, 4010, 64, 3, 6, 128, head_dim=128, form="many"),
    beside("many_in_turns_small", 2048, 40000, 1700, 30, 1, 3, 256, heads=1, frame=4, form="many small"),
    case("many_in_turns_70", [16384, 5000] + [3] * 70, [3000 * 32, 30] + [1] * 70, heads=1, gone=[(0, 0, 16384)] + between(256, 6, 5), of=1,
         rows_chunks=6, keys_chunks=12, form="many"),
    # pieces bounded by the workspace: 2^21 rows, most of them of a sequence without keys
    case("many_few_pieces", [0, 12000], [(1 << 20) - 40, 40], heads=2, kv_heads=1, gone=between(256, 3, 16), frame=13, dtypes=("e2m1",), of=1,
         form="many small", rows_chunks=3, keys_chunks=1, tokens=1 << 20),
]


class Shared(Pool):
    """`kind`: "random"; "stairs": levels that rise and fall from tile to tile, by sums that have to raise their reference; "high", "low":
    scores close to 2^28 or to -2^28 that differ by 16 and 32."""

    def __init__(self, c, dtype, kind, seed=50, distinct=24):
        page, n = c["page"], 3 if c["page"] == 1024 else distinct
        super().__init__(seed, [n * page], dtype=dtype, heads=c["heads"], kv_heads=c["kv_heads"], head_dim=c["head_dim"], page=page, spare=0,
                         scale=0.0 if kind == "random" else 1.0)
        self.c, self.kind, self.lens = c, kind, c["lens"]
        rng = self.rng
        if kind != "random":
            self.fill(kind)
        n_seq, columns = len(self.lens), c["columns"]
        self.table = np.full((n_seq, columns), -1, np.int32)
        for s, length in enumerate(self.lens):
            used = -(-length // page)
            ids = rng.integers(0, self.n_pages, used)
            if kind == "stairs":       # pages j, j + 3, .. are of level j; a tile of 32 keys is of one
                tile = np.arange(used) * min(page, 32) // 32
                ids = ids // 3 * 3 + (tile * 7 + tile // 5) % 3
            self.table[s, :used] = ids
        for s, a, b in c["gone"]:
            self.table[s, a // page:-(-b // page)] = -1
        self.max_pages = columns
        self.p = B.make_cache_params(n_seq, c["heads"], c["head_dim"], kv_heads=c["kv_heads"], cache_dtype=DTYPES[dtype], page_tokens=page,
                                     n_pages=self.n_pages, max_pages=columns, frame_tokens=c["frame"], softmax_scale=self.scale)
        self.o.table = self.table
        self.d = self.device()

    def fill(self, kind):
        k = np.zeros_like(self.o.k)
        at = np.arange(self.p.page_tokens)
        if kind == "stairs":
            k[..., 0] = (np.arange(self.n_pages) % 3 * LEVEL)[:, None, None]
            k[..., 32] = np.array([0, 0.5, 1, 0.25, 0.75, 1.5, 2])[at % 7]
        else:
            k[..., 0] = 1.5 * 2.0 ** 13
            k[..., 32] = at % 3
        if self.dtype == "e2m1":       # (three kinds of pages, all heads alike)
            some = S.round_blocks(k[:3, :1])
            for name, x in zip(("k", "ke", "kc"), some):
                setattr(self.o, name, np.tile(x, (len(k) // 3, k.shape[1], 1, 1)))
        elif self.dtype == "e4m3":
            self.o.ke = np.full(self.o.ke.shape, 0 if kind == "stairs" else 5)
            self.o.k = k
        else:
            self.o.k = k
        assert np.array_equal(self.o.k, k)

    def queries(self):
        """[tokens, heads, d] on the device; rows of no interest (of the sequence that holds nothing) are zeros."""
        c = self.c
        n = c["tokens"] or sum(c["new"])
        shown = min(n, 6000)
        q = np.zeros((shown, c["heads"], c["head_dim"]))
        if self.kind == "random":
            q = rows(self.rng, shown, c["heads"], c["head_dim"])
        elif self.kind == "stairs":
            q[..., 0] = np.where(np.arange(shown) % 4 == 3, 0.5, 1.0)[:, None]
            q[..., 32] = 1.0 + np.arange(c["heads"]) % 2
        else:
            q[..., 0] = 1.25 * 2.0 ** 14 * (1 if self.kind == "high" else -1)
            q[..., 32] = 16.0
        out = torch.zeros(n, c["heads"], c["head_dim"], dtype=torch.bfloat16, device="cuda")
        out[n - shown:] = dev(q)
        return out

    def exact_drawn(self, q):
        """[n_seq, kv_heads, positions] in 64 bits, and which are held."""
        c, p = self.c, self.p
        room, group = self.max_pages * c["page"], c["heads"] // c["kv_heads"]
        out = torch.zeros(len(self.lens), c["kv_heads"], room, dtype=torch.float64, device="cuda")
        held = torch.zeros(len(self.lens), room, dtype=torch.bool, device="cuda")
        k_all = torch.from_numpy(self.o.k).cuda()
        at = 0
        for s, (new, length) in enumerate(zip(c["new"], self.lens)):
            t = torch.arange(length, device="cuda")
            ids = torch.from_numpy(self.table[s]).cuda().long()[t // c["page"]]
            held[s, :length] = ids >= 0
            if new and bool((ids >= 0).any()):
                k = k_all[ids.clamp(min=0), :, t % c["page"]]
                limit = torch.full((new,), length, device="cuda")
                if c["frame"]:
                    pos = torch.arange(length - new, length, device="cuda")
                    limit = torch.where(pos < 0, 0, (torch.div(pos, c["frame"], rounding_mode="floor") + 1) * c["frame"])
                shut = ~((ids >= 0) & (t < limit[:, None]))
                for h in range(c["heads"]):
                    z = q[at:at + new, h].double() @ k[:, h // group].t().contiguous() * self.softmax_scale()
                    z.masked_fill_(shut, -torch.inf)
                    top = z.amax(1, keepdim=True)
                    w = torch.exp(z - torch.where(torch.isfinite(top), top, 0.0))
                    total = w.sum(1, keepdim=True)
                    out[s, h // group, :length] += (w / torch.where(total > 0, total, 1.0)).sum(0)
            at += new
        return out, held

    def check(self):
        c, p = self.c, self.p
        q = self.queries()
        n = q.shape[0]
        off = [0] + np.cumsum(c["new"]).tolist()
        shape = (p.n_seq, p.kv_heads, p.max_pages * p.page_tokens)
        had = torch.rand(shape, device="cuda") * 1e-3
        out = torch.full(shape, 5.0, device="cuda")
        ws = B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, n)).fill_(255)
        B.litevggt_cached_mass(p, self.d, q, i32(off), i32(self.lens), had, out, ws)
        drawn, held = self.exact_drawn(q)
        length = torch.tensor(self.lens, device="cuda")
        inside = (torch.arange(shape[2], device="cuda") < length[:, None])[:, None].expand(shape)
        assert (out[~inside] == 5.0).all()
        exact = torch.where(held[:, None], had.double() + drawn, 0.0)
        # A score's error (exact in the kinds that are made up) is its weight's and its row's; exp2 and its argument, of weights down to e^-80:
        # 2^-17 + 80 * 2^-22; chains of sums: 1024 within and over the pieces of a row, one for each row of a key
        error = 0.0
        if self.kind == "random":
            k = self.o.k
            norm = float(q.double().square().sum(-1).max().sqrt()) * np.sqrt((k ** 2).sum(-1)).max()
            error = self.softmax_scale() * p.head_dim * 2.0 ** -24 * norm
        rows_of = max(c["new"][c["of"]], 32) * p.heads // p.kv_heads
        rel = 2 * error + 2.0 ** -17 + 80 * 2.0 ** -22 + (1024 + rows_of) * 2.0 ** -24
        if self.kind in ("high", "low"):
            rel += 2.0 ** -18       # the reference is off by half a step, 16 here: arguments up to 16 + 32 log2(e) in magnitude, off by 2^-19
        tol = rel * drawn + 2.0 ** -23 * exact + 1e-30
        assert bool(torch.isfinite(out).all())
        bad = ((out - exact).abs() > tol) & inside
        assert not bool(bad.any()), (torch.nonzero(bad)[:5].tolist(), float(((out - exact).abs() / tol)[inside].max()))
        return out
