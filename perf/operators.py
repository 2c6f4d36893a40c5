"""What is measured of the operators that serve frames as they arrive: the paged cache of K and V that is quantised as it is
written and read back, the attention of new tokens over it, and cross attention to states of another length.

``run`` computes them in plain torch where ``own`` is false, through the package where it is true.  Shapes are the package's
own where it has them (frames of 37 x 37 patches and 5 special tokens = 1374 tokens, 16 heads of 64; frames of 16 x 16 = 261
tokens, 4 heads) and generic otherwise.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6          # of the RMS normalisation of q and k
FP8_MAX = 448.0
HEADROOM = 3        # pages of the pool that belong to nobody in the call


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a single new token's K and V go into the cache: launch latency
        _write("write_one_token", 1, 1, 1, heads=16, dim=64, dtype="bf16", page=64, held=(500, 500)),
        # eight streams append four frames each, K and V out of one projection's output
        _write("write_frames_e4m3", 8, 5496, 5496, heads=16, dim=64, dtype="e4m3", page=128, held=(1374, 13740), fused=True),
        # the whole cache of a hundred frames handed to a consumer that wants rows
        _read("read_100_frames_e4m3", 1, 137400, 137400, heads=16, dim=64, dtype="e4m3", page=128),
        # short ragged ranges out of small pages
        _read("read_ragged_bf16", 7, 90, 1203, heads=4, dim=128, dtype="bf16", page=16),
        # the smallest step: one token over a short cache
        _cached("token_short", 1, 1, 1, 394, 394, heads=4, kv=4, dim=64, dtype="bf16", page=64, frame=1),
        # a batch of single tokens over caches of very different lengths, heads shared
        _cached("tokens_ragged_e4m3", 32, 1, 1, 301, 30011, heads=16, kv=4, dim=128, dtype="e4m3", page=16, frame=1),
        # the five special tokens of a new frame over a hundred frames
        _cached("specials_long", 1, 5, 5, 137405, 137405, heads=16, kv=16, dim=64, dtype="bf16", page=64, frame=0),
        # a whole new frame over a hundred frames
        _cached("frame_over_100", 1, 1374, 1374, 138774, 138774, heads=16, kv=16, dim=64, dtype="bf16", page=128, frame=1374),
        # chunks of several frames, each seeing the frames up to its own, some pages given back
        _cached("chunks_ragged_e4m3", 6, 261, 2088, 2349, 20097, heads=16, kv=16, dim=64, dtype="e4m3", page=32, frame=261,
                norm=True, evicted=7),
        # special tokens over one frame's states
        _cross("cross_small", 2, 5, 5, 1374, 1374, heads=16, kv=16, dim=64),
        # ten frames' tokens over a merged sequence
        _cross("cross_frames", 1, 13740, 13740, 14316, 14316, heads=16, kv=16, dim=64, fused=True),
        # ragged sets over ragged states, one of them empty, heads shared, normalised
        _cross("cross_ragged", 9, 3, 701, 0, 6007, heads=16, kv=2, dim=128, norm=True),
    ]


def draw(rng):
    most = [max(v) for v in zip(*(_costs(c) for c in listed()))]
    while True:
        case = _drawn(rng)
        if all(a <= b for a, b in zip(_costs(case), most)):
            return case


def _drawn(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["write", "read", "cached", "cached", "cross"])
    dim = rng.choice([64, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 16])
    page = rng.choice([16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "e4m3"])
    n_seq = rng.choice([1, 1, 2, 3, 5, 8, 17, 40])
    if op == "write":
        most = log_int(1, 44000 // n_seq + 1)
        held = log_int(1, 20000 // n_seq + 1)
        return _write(None, n_seq, max(1, most // rng.choice([1, 1, 3])), most, heads=kv, dim=dim, dtype=dtype, page=page,
                      held=(held // 2, held), fused=rng.random() < 0.5, norm=rng.random() < 0.3, evicted=rng.choice([0, 0, 5]))
    if op == "read":
        most = log_int(1, 130000 // n_seq + 1)
        return _read(None, n_seq, max(1, most // rng.choice([1, 2, 9])), most, heads=kv, dim=dim, dtype=dtype, page=page,
                     evicted=rng.choice([0, 0, 5]))
    group = rng.choice([1, 1, 2, 4, 8])
    heads = min(kv * group, 32) // kv * kv
    if op == "cached":
        most = rng.choice([1, 1, log_int(1, 64), log_int(16, 6000)])
        least = max(1, most // rng.choice([1, 1, 4]))
        held = log_int(1, 140000)
        frame = rng.choice([0, 1, 1, 261, 1374])
        return _cached(None, n_seq, least, most, held // rng.choice([1, 2, 30]) + most, held + most, heads=heads, kv=kv, dim=dim,
                       dtype=dtype, page=page, frame=frame, norm=rng.random() < 0.3, evicted=rng.choice([0, 0, 0, 9]))
    most = log_int(1, 14000)
    states = log_int(1, 40000)
    return _cross(None, n_seq, max(1, most // rng.choice([1, 1, 5])), most, states // rng.choice([1, 1, 2, 50]), states, heads=heads,
                  kv=kv, dim=dim, fused=rng.random() < 0.5, norm=rng.random() < 0.3)


def _case(name, **kw):
    return {**({"name": name} if name else {}), **kw}


def _write(name, n_seq, lo, hi, *, heads, dim, dtype, page, held, fused=False, norm=False, evicted=0):
    """Chunks of lo..hi new tokens go behind held tokens."""
    return _case(name, op="write", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=heads, head_dim=dim, dtype=dtype,
                 page=page, len_lo=held[0], len_hi=held[1], fused=fused, norm=norm, evicted=evicted, frame=0)


def _read(name, n_seq, lo, hi, *, heads, dim, dtype, page, evicted=0):
    """The first lo..hi tokens of each sequence."""
    return _case(name, op="read", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=heads, head_dim=dim, dtype=dtype,
                 page=page, len_lo=lo, len_hi=hi, fused=False, norm=False, evicted=evicted, frame=0)


def _cached(name, n_seq, lo, hi, len_lo, len_hi, *, heads, kv, dim, dtype, page, frame, norm=False, evicted=0):
    """lo..hi new tokens, the last ones of the len_lo..len_hi that the cache holds."""
    return _case(name, op="cached", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=kv, head_dim=dim, dtype=dtype,
                 page=page, len_lo=len_lo, len_hi=len_hi, fused=False, norm=norm, evicted=evicted, frame=frame)


def _cross(name, n_seq, lo, hi, len_lo, len_hi, *, heads, kv, dim, fused=False, norm=False):
    """lo..hi queries over len_lo..len_hi states."""
    return _case(name, op="cross", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=kv, head_dim=dim, dtype="bf16",
                 page=0, len_lo=len_lo, len_hi=len_hi, fused=fused, norm=norm, evicted=0, frame=0)


def _spread(lo, hi, n, phase):
    """n whole numbers between lo and hi in no order, the first two the limits."""
    if n == 1:
        return [hi]
    return [lo, hi][:n] + [lo + int((hi - lo) * ((phase + 0.6180339887 * i) % 1.0)) for i in range(2, n)]


def _sizes(case):
    """(new tokens, held tokens) of each sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["n_seq"], 0.3)
    if case["op"] == "read":
        return new, new
    held = _spread(case["len_lo"], case["len_hi"], case["n_seq"], 0.7)
    if case["op"] == "cached":
        held = [max(a, b) for a, b in zip(held, new)]
    return new, held


def _visible(case, n, length):
    """Keys that the n queries of a sequence see, summed over the queries."""
    if not case["frame"]:
        return n * length
    T, total, p = case["frame"], 0, length - n
    while p < length:   # a frame's queries at a time
        end = min((p // T + 1) * T, length)
        total += (end - p) * end
        p = end
    return total


def work(case):
    new, held = _sizes(case)
    d, kv, heads = case["head_dim"], case["kv_heads"], case["heads"]
    n = sum(new)
    row = kv * (d * 2 if case["dtype"] == "bf16" else d + 1)     # K or V of one token in the cache
    if case["op"] in ("write", "read"):
        return {"bytes": 2.0 * n * (kv * d * 2 + row), "flops": 0.0}
    if case["op"] == "cross":
        return {"bytes": 2.0 * 2 * n * heads * d + 2.0 * sum(held) * kv * d * 2,
                "flops": 4.0 * sum(a * b for a, b in zip(new, held)) * heads * d}
    return {"bytes": 2.0 * 2 * n * heads * d + 2.0 * sum(held) * row,
            "flops": 4.0 * sum(_visible(case, a, b) for a, b in zip(new, held)) * heads * d}


def _costs(case):
    """Bytes, flops, and about how long the plain form takes, whose scores are written and read several times."""
    w = work(case)
    new, held = _sizes(case)
    scores = sum(a * b for a, b in zip(new, held)) * case["heads"] if case["op"] in ("cached", "cross") else 0
    return w["bytes"], w["flops"], w["bytes"] / 4e12 + w["flops"] / 5e13 + scores * 40.0 / 4e12 + len(new) * 2e-4


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    new, held = _sizes(case)
    n, n_seq, kv, heads, d = sum(new), case["n_seq"], case["kv_heads"], case["heads"], case["head_dim"]

    def offsets(v):
        return torch.tensor([0] + torch.tensor(v).cumsum(0).tolist(), dtype=torch.int32)

    def rows(count, width):
        return torch.randn(count, width, generator=g, device=DEV, dtype=torch.bfloat16)

    def key_values(count):
        """K and V of `count` tokens, channels of unlike sizes, as slices of one projection's output or apart."""
        gain = torch.exp(0.5 * torch.randn(kv * d, generator=g, device=DEV)).to(torch.bfloat16)
        if case["fused"]:
            both = rows(count, 2 * kv * d)
            both[:, :kv * d] *= gain
            return both[:, :kv * d].unflatten(1, (kv, d)), both[:, kv * d:].unflatten(1, (kv, d))
        return (rows(count, kv * d) * gain).unflatten(1, (kv, d)), rows(count, kv * d).unflatten(1, (kv, d))

    s = {"case": case, "new": new, "held": held, "new_off": offsets(new).to(DEV)}
    if case["op"] in ("cached", "cross"):
        s["q"] = rows(n, heads * d).unflatten(1, (heads, d))
        s["o"] = torch.empty_like(s["q"])
    if case["op"] == "cross":
        s["k"], s["v"] = key_values(sum(held))
        off = offsets(held).to(DEV)
        s["kv_begin"], s["kv_end"] = off[:-1].contiguous(), off[1:].contiguous()
        return s

    # the pool: every sequence's pages somewhere in it, some given back
    page = case["page"]
    total = [a + b for a, b in zip(new, held)] if case["op"] == "write" else held
    pages = [-(-t // page) for t in total]
    n_pages, max_pages = sum(pages) + HEADROOM, max(pages)
    where = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((n_seq, max_pages), -1, dtype=torch.int32)
    at = 0
    for i, c in enumerate(pages):
        table[i, :c] = where[at:at + c]
        at += c
    if case["evicted"]:      # every so many pages, but for a sequence's last one
        for i, c in enumerate(pages):
            table[i, case["evicted"] // 2:max(c - 1, 0):case["evicted"]] = -1
    s.update(n_pages=n_pages, max_pages=max_pages, table=table.to(DEV),
             held_dev=torch.tensor(held, dtype=torch.int32, device=DEV), zero=torch.zeros(n_seq, dtype=torch.int32, device=DEV))
    shape = (n_pages, kv, page, d)
    if case["op"] == "write":
        s["k"], s["v"] = key_values(n)
        kind = torch.bfloat16 if case["dtype"] == "bf16" else torch.uint8
        s["pool_k"], s["pool_v"] = (torch.zeros(shape, dtype=kind, device=DEV) for _ in range(2))
        s["scale_k"], s["scale_v"] = (torch.zeros(shape[:3], dtype=torch.uint8, device=DEV) for _ in range(2))
        return s
    gain = torch.exp(0.5 * torch.randn(kv, 1, d, generator=g, device=DEV))
    for name, by in (("k", gain), ("v", None)):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        if by is not None:
            x *= by.to(torch.bfloat16)
        if case["dtype"] == "e4m3":
            code, e = _quantised(x)
            s["pool_" + name], s["scale_" + name] = code.view(torch.uint8), e
        else:
            s["pool_" + name], s["scale_" + name] = x, torch.zeros(shape[:3], dtype=torch.uint8, device=DEV)
    if case["op"] == "read":
        s["out_k"], s["out_v"] = (torch.empty(n, kv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2512_04939_amd import binding as B

    case = s["case"]
    if "params" not in s:      # what a program makes once for its shapes
        if case["op"] == "cross":
            s["params"] = B.make_cross_params(case["n_seq"], case["heads"], case["head_dim"], kv_heads=case["kv_heads"],
                                              qk_norm=int(case["norm"]))
            s["ws"] = B.alloc_ws(B.litevggt_cross_attn_ws_bytes(s["params"], s["q"].shape[0], s["k"].shape[0]))
        else:
            s["params"] = B.make_cache_params(case["n_seq"], case["heads"], case["head_dim"], kv_heads=case["kv_heads"],
                                              cache_dtype=B.CACHE_BF16 if case["dtype"] == "bf16" else B.CACHE_E4M3,
                                              page_tokens=case["page"], n_pages=s["n_pages"], max_pages=s["max_pages"],
                                              frame_tokens=case["frame"], qk_norm=int(case["norm"]))
            s["cache"] = B.CacheBuffers(s["pool_k"], s["pool_v"], s["scale_k"], s["scale_v"], s["table"])
            if case["op"] == "cached":
                s["ws"] = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(s["params"], s["q"].shape[0]))
    p = s["params"]
    if case["op"] == "write":
        B.litevggt_cache_write(p, s["cache"], s["k"], s["v"], s["new_off"], s["held_dev"])
        return _held(s)
    if case["op"] == "read":
        B.litevggt_cache_read(p, s["cache"], s["zero"], s["new_off"], s["out_k"], s["out_v"])
        return s["out_k"], s["out_v"]
    if case["op"] == "cached":
        B.litevggt_cached_attn(p, s["cache"], s["q"], s["new_off"], s["held_dev"], s["o"], s["ws"])
    else:
        B.litevggt_cross_attn(p, s["q"], s["new_off"], s["k"], s["v"], s["kv_begin"], s["kv_end"], s["o"], s["ws"])
    return s["o"]


def _held(s):
    """The whole pool: as it is, or its codes' values and its exponents."""
    if s["case"]["dtype"] == "bf16":
        return s["pool_k"], s["pool_v"]
    return tuple(s[k].view(torch.float8_e4m3fn) for k in ("pool_k", "pool_v")) + (s["scale_k"], s["scale_v"])


def _quantised(x):
    """E4M3 codes and biased exponents of rows x [..., d]."""
    f = x.float()
    a = torch.where(torch.isfinite(f), f.abs(), 0.0).amax(-1)
    m, e = torch.frexp(a)                                    # a = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(a > 0, e - 9 + (m > 0.875).int(), 0).clamp(min=-126)
    code = (f * _two_to(-e[..., None])).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
    return code, (e + 127).to(torch.uint8)


def _two_to(e):
    """2^e from its bits: pow may be an ulp off, which moves values on the border of two codes."""
    return (e.int() + 127 << 23).view(torch.float32)


def _normed(x):
    f = x.float()
    return (f / torch.sqrt(f.square().mean(-1, keepdim=True) + EPS)).to(x.dtype)


def _at(s, i, first, count):
    """Pages and places in them of positions first .. first + count - 1 of sequence i; a page of -1: not held."""
    pos = torch.arange(first, first + count, device=DEV)
    return s["table"][i, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _rows_of(s, name, page, place):
    """Rows of the cache in 32 bits, zeros where a page is not held."""
    x = s["pool_" + name][page.clamp(min=0), :, place]
    if s["case"]["dtype"] == "e4m3":
        x = x.view(torch.float8_e4m3fn).float() * _two_to(s["scale_" + name][page.clamp(min=0), :, place].int()[..., None] - 127)
    return torch.where((page >= 0)[:, None, None], x.float(), 0.0)


def _softmax_sum(case, q, k, v, seen):
    """q [n, heads, d], k and v [m, kv, d] in 32 bits, seen [n, m] or None -> [n, heads, d]."""
    n, heads, d = q.shape
    kv = k.shape[1]
    rows = q.unflatten(1, (kv, heads // kv)).permute(1, 2, 0, 3).reshape(kv, heads // kv * n, d)
    w = torch.bmm(rows, k.permute(1, 2, 0).contiguous()).mul_(1.0 / math.sqrt(d)).unflatten(1, (heads // kv, n))
    if seen is not None:
        w.masked_fill_(~seen, -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(torch.where(torch.isfinite(top), top, 0.0)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.bmm(w.flatten(1, 2), v.transpose(0, 1).contiguous()).unflatten(1, (heads // kv, n))
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(2, 0, 1, 3).reshape(n, heads, d)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "write":
        return _write_plain(s)
    if case["op"] == "read":
        page, place = (torch.cat(v) for v in zip(*(_at(s, i, 0, c) for i, c in enumerate(s["new"]))))
        return tuple(_rows_of(s, name, page, place).to(torch.bfloat16) for name in ("k", "v"))
    out = []
    at = states = 0
    for i, (n, m) in enumerate(zip(s["new"], s["held"])):
        q = s["q"][at:at + n]
        q = (_normed(q) if case["norm"] else q).float()
        at += n
        seen = None
        if case["op"] == "cross":
            k, v = s["k"][states:states + m], s["v"][states:states + m]
            k, v = (_normed(k) if case["norm"] else k).float(), v.float()
            states += m
        else:
            page, place = _at(s, i, 0, m)
            k, v = _rows_of(s, "k", page, place), _rows_of(s, "v", page, place)
            if case["frame"] or case["evicted"]:
                t, p = torch.arange(m, device=DEV), torch.arange(m - n, m, device=DEV)
                T = case["frame"] or m
                seen = (page >= 0)[None, :] & (t[None, :] < ((p // T + 1) * T)[:, None])
        out.append(_softmax_sum(case, q, k, v, seen) if m else torch.zeros_like(q))
    return torch.cat(out).to(torch.bfloat16)


def _write_plain(s):
    page, place = (torch.cat(v) for v in zip(*(_at(s, i, h, c) for i, (c, h) in enumerate(zip(s["new"], s["held"])))))
    held = page >= 0
    for name in ("k", "v"):
        x = _normed(s["k"]) if name == "k" and s["case"]["norm"] else s[name]
        if s["case"]["dtype"] == "e4m3":
            x, e = _quantised(x)
            s["scale_" + name][page[held], :, place[held]] = e[held]
            x = x.view(torch.uint8)
        s["pool_" + name][page[held], :, place[held]] = x[held]
    return _held(s)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    scores = sum(a * b for a, b in zip(s["new"], s["held"])) * case["heads"]
    if case["op"] in ("cached", "cross") and scores * case["head_dim"] > 3e12:
        return None
    norm = lambda x: (x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()).to(torch.bfloat16).double()   # noqa: E731
    if case["op"] == "write":
        return _exact_write(s, norm)
    value = lambda name: _exact_pool(s, name)                                                             # noqa: E731
    if case["op"] == "read":
        pools = [value("k"), value("v")]
        return tuple(torch.cat([_exact_rows(s, x, i, c) for i, c in enumerate(s["new"])]) for x in pools)
    n, heads, d = s["q"].shape
    group = heads // case["kv_heads"]
    out = torch.zeros(n, heads, d, dtype=torch.float64, device=DEV)
    pools = None if case["op"] == "cross" else [value("k"), value("v")]
    ends = torch.tensor(s["new"]).cumsum(0).tolist()
    for i, (c, m) in enumerate(zip(s["new"], s["held"])):
        if m == 0:
            continue
        q = s["q"][ends[i] - c:ends[i]].double()
        if case["norm"]:
            q = norm(q)
        if pools is None:
            lo = sum(s["held"][:i])
            k, v = s["k"][lo:lo + m].double(), s["v"][lo:lo + m].double()
            if case["norm"]:
                k = norm(k)
            there = torch.ones(m, dtype=torch.bool, device=DEV)
        else:
            k, v = (_exact_rows(s, x, i, m) for x in pools)
            there = s["table"][i].repeat_interleave(case["page"])[:m] >= 0
        t = torch.arange(m, device=DEV)
        limit = torch.full((c,), m, device=DEV)
        if case["frame"]:
            limit = (torch.arange(m - c, m, device=DEV) // case["frame"] + 1) * case["frame"]
        for b in range(0, c, 512):
            shut = ~(there & (t < limit[b:b + 512, None]))
            for h in range(heads):
                z = q[b:b + 512, h] @ k[:, h // group].t().contiguous() / math.sqrt(d)
                z[shut] = -math.inf
                best = z.max(1, keepdim=True).values
                w = torch.exp(z - torch.where(best == -math.inf, 0.0, best))
                norm_of = w.sum(1, keepdim=True)
                out[ends[i] - c + b:ends[i] - c + b + w.shape[0], h] = (w / torch.where(norm_of == 0, 1.0, norm_of)) @ v[:, h // group].contiguous()
    return out


def _exact_pool(s, name):
    x = s["pool_" + name]
    if s["case"]["dtype"] == "bf16":
        return x
    return x, s["scale_" + name]


def _exact_rows(s, pool, i, count):
    """The first `count` positions of sequence i, a page at a time."""
    page = s["case"]["page"]
    ids = s["table"][i, :-(-count // page)].long()
    codes, e = (pool, None) if torch.is_tensor(pool) else pool
    x = codes[ids.clamp(min=0)].transpose(1, 2)                       # [pages, places, kv, d]
    if e is None:
        x = x.double()
    else:
        power = (e[ids.clamp(min=0)].transpose(1, 2).long() + (1023 - 127) << 52).view(torch.float64)
        x = x.contiguous().view(torch.float8_e4m3fn).double() * power[..., None]
    x[ids < 0] = 0.0
    return x.reshape(-1, *x.shape[2:])[:count]


def _exact_write(s, norm):
    case, page = s["case"], s["case"]["page"]
    pools = [s["pool_k"], s["pool_v"], s["scale_k"], s["scale_v"]]
    flat = [p.transpose(1, 2).reshape(-1, *p.shape[1:2], *p.shape[3:]) for p in pools]   # [pages * places, kv, ..]
    flat = [f.double() if f.dtype == torch.bfloat16 else f for f in flat]
    codes = [torch.zeros(f.shape, dtype=torch.float64, device=DEV) for f in flat[:2]]
    start = 0
    for i, (c, h) in enumerate(zip(s["new"], s["held"])):
        pos = torch.arange(h, h + c, device=DEV)
        ids = s["table"][i][torch.div(pos, page, rounding_mode="floor")].long()
        keep = (ids >= 0).nonzero().squeeze(1)
        to = ids[keep] * page + pos[keep] % page
        for j, name in enumerate(("k", "v")):
            x = s[name][start:start + c][keep].double()
            if case["norm"] and name == "k":
                x = norm(x)
            if case["dtype"] == "bf16":
                flat[j][to] = x
                continue
            a = x.abs().amax(-1)
            e = torch.ceil(torch.log2(a.clamp(min=1e-300) / FP8_MAX))
            power = lambda y: (y.long() + 1023 << 52).view(torch.float64)                  # noqa: E731
            e = e + (a > FP8_MAX * power(e)).double() - (a <= FP8_MAX * power(e - 1)).double()
            e = torch.where(a > 0, e, 0.0).clamp(min=-126)
            z = x / power(e)[..., None]
            step = power(torch.frexp(z.abs().clamp(min=2.0 ** -6)).exponent - 4)           # spacing of E4M3 at z
            codes[j][to] = torch.round(z / step) * step
            flat[2 + j][to] = (e + 127).to(torch.uint8)
        start += c
    back = lambda f: f.reshape(-1, page, *f.shape[1:]).transpose(1, 2)                    # noqa: E731
    if case["dtype"] == "bf16":
        return tuple(back(f) for f in flat[:2])
    return tuple(back(f) for f in codes + flat[2:])
