"""What is measured of the operators that keep a stream's cache small: rotary positions with several axes for what goes into it, K
and V held in 4 bits and attention over them, the attention weight that each held position has drawn, and the eviction of the
pages that drew the least.

``run`` computes them in plain torch where ``own`` is false, through the package where it is true.  Shapes are the package's
own where it has them (frames of 37 x 37 patches and 5 special tokens = 1374 tokens, 16 heads of 64; frames of 16 x 16 = 261
tokens, 4 heads) and generic otherwise.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6          # of the RMS normalisation of q and k
HEADROOM = 3        # pages of the pool that belong to nobody in the call
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MOST = 6.0          # its largest value
BLOCK = 32          # channels that share a scale


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a single new token's q and k: launch latency
        _rope("rope_one_token", 1, heads=16, kv=16, dim=64, pairs=(16, 16), pairing="axis", joint=False, base=100.0, far=40),
        # 32 frames, rows and columns of their patches, q and k out of one projection's output
        _rope("rope_frames", 43968, heads=16, kv=16, dim=64, pairs=(16, 16), pairing="axis", joint=False, base=100.0, far=40, fused=True),
        # the gradient for a video's tokens: time, height and width, times far from the start, heads shared
        _rope("rope_video_gradient", 20011, heads=16, kv=4, dim=128, pairs=(16, 24, 24), pairing="head", joint=True, base=10000.0,
              far=1000003, inverse=True),
        # a new token of each of two streams is stored and read back
        _store("store_two_tokens", 2, 1, 1, kv=16, dim=64, page=64, held=(499, 500)),
        # eight streams store four frames each, K and V out of one projection's output, and hand them to a consumer that wants rows
        _store("store_frames", 8, 5496, 5496, kv=16, dim=64, page=128, held=(1374, 13740), fused=True),
        # a batch of single tokens over caches of very different lengths, heads shared
        _attn("tokens_ragged", 32, 1, 1, 301, 30011, heads=16, kv=4, dim=128, page=16, frame=1),
        # a whole new frame over a hundred frames
        _attn("frame_over_100", 1, 1374, 1374, 138774, 138774, heads=16, kv=16, dim=64, page=128, frame=1374),
        # chunks of several frames, each seeing the frames up to its own, some pages given back
        _attn("chunks_ragged", 6, 261, 2088, 2349, 20097, heads=16, kv=16, dim=64, page=32, frame=261, norm=True, evicted=7),
        # what the special tokens of a new frame look at in a hundred frames
        _mass("mass_specials", 1, 5, 5, 137405, 137405, heads=16, kv=16, dim=64, dtype="bf16", page=64, frame=0),
        # what whole new frames of four streams look at, some pages given back
        _mass("mass_frames", 4, 1374, 1374, 2748, 41220, heads=16, kv=16, dim=64, dtype="e2m1", page=32, frame=1374, evicted=9),
        # a short cache loses a few pages
        _evict("evict_short", 1, 394, 394, kv=4, page=16, keep=0.7, first=1, last=2),
        # many streams lose a third of their pages, small ones, but for their first frame's and their last one's
        _evict("evict_streams", 32, 13740, 137400, kv=16, page=16, keep=0.66, first=86, last=86, evicted=11),
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

    op = rng.choice(["rope", "store", "attn", "attn", "mass", "evict"])
    dim = rng.choice([64, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 16])
    heads = min(kv * rng.choice([1, 1, 2, 4, 8]), 32) // kv * kv
    page = rng.choice([16, 32, 64, 128, 256])
    n_seq = rng.choice([1, 1, 2, 3, 5, 8, 17, 40])
    evicted = rng.choice([0, 0, 0, 5, 9])
    if op == "rope":
        axes = rng.choice([1, 2, 2, 3, 3, 4])
        pairs = [max(1, dim // 2 // axes // rng.choice([1, 1, 2])) for _ in range(axes)]
        pairs[-1] = rng.choice([pairs[-1], dim // 2 - sum(pairs[:-1])])
        return _rope(None, log_int(1, 60000), heads=heads, kv=rng.choice([kv, kv, 0]), dim=dim, pairs=tuple(pairs),
                     pairing=rng.choice(["axis", "head", "adjacent"]), joint=rng.random() < 0.5, base=rng.choice([100.0, 10000.0, 500000.0]),
                     far=log_int(2, 2000000), fused=rng.random() < 0.5, inverse=rng.random() < 0.4)
    if op == "store":
        most = log_int(1, 44000 // n_seq + 1)
        held = log_int(1, 20000 // n_seq + 1)
        return _store(None, n_seq, max(1, most // rng.choice([1, 1, 3])), most, kv=kv, dim=dim, page=page, held=(held // 2, held),
                      fused=rng.random() < 0.5, evicted=evicted)
    if op == "evict":
        held = log_int(1, 140000)
        return _evict(None, n_seq, max(1, held // rng.choice([1, 3, 20])), held, kv=kv, page=page, keep=rng.choice([0.0, 0.3, 0.66, 0.95, 1.2]),
                      first=rng.choice([0, 1, 5]), last=rng.choice([0, 1, 9]), evicted=evicted)
    most = rng.choice([1, 1, log_int(1, 64), log_int(16, 6000)])
    least = max(1, most // rng.choice([1, 1, 4]))
    held = log_int(1, 140000)
    frame = rng.choice([0, 1, 1, 261, 1374])
    lengths = (held // rng.choice([1, 2, 30]) + most, held + most)
    if op == "attn":
        return _attn(None, n_seq, least, most, *lengths, heads=heads, kv=kv, dim=dim, page=page, frame=frame, norm=rng.random() < 0.3,
                     evicted=evicted)
    return _mass(None, n_seq, least, most, *lengths, heads=heads, kv=kv, dim=dim, dtype=rng.choice(["bf16", "e4m3", "e2m1"]), page=page,
                 frame=frame, evicted=evicted)


def _case(name, **kw):
    base = dict(n_seq=1, new_lo=0, new_hi=0, len_lo=0, len_hi=0, heads=0, kv_heads=0, head_dim=0, dtype="e2m1", page=0, frame=0,
                fused=False, norm=False, evicted=0)
    return {**({"name": name} if name else {}), **base, **kw}


def _rope(name, n, *, heads, kv, dim, pairs, pairing, joint, base, far, fused=False, inverse=False):
    """n tokens at positions up to `far` on the first axis, of a frame's size on the others; pairs of channels by axis."""
    three = list(pairs) + [0] * (4 - len(pairs))
    return _case(name, op="rope", new_lo=n, new_hi=n, heads=heads, kv_heads=kv, head_dim=dim, axes=len(pairs), pairs0=three[0], pairs1=three[1],
                 pairs2=three[2], pairs3=three[3], pairing=pairing, joint=joint, base=base, far=far, fused=fused, inverse=inverse)


def _store(name, n_seq, lo, hi, *, kv, dim, page, held, fused=False, evicted=0):
    """Chunks of lo..hi new tokens go behind held tokens and are read back."""
    return _case(name, op="store", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=kv, kv_heads=kv, head_dim=dim, page=page,
                 len_lo=held[0], len_hi=held[1], fused=fused, evicted=evicted)


def _attn(name, n_seq, lo, hi, len_lo, len_hi, *, heads, kv, dim, page, frame, norm=False, evicted=0):
    """lo..hi new tokens, the last ones of the len_lo..len_hi that the cache holds."""
    return _case(name, op="attn", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=kv, head_dim=dim, page=page, len_lo=len_lo,
                 len_hi=len_hi, norm=norm, evicted=evicted, frame=frame)


def _mass(name, n_seq, lo, hi, len_lo, len_hi, *, heads, kv, dim, dtype, page, frame, evicted=0):
    """The weight that lo..hi new tokens give each of the len_lo..len_hi positions, on top of what these had."""
    return _case(name, op="mass", n_seq=n_seq, new_lo=lo, new_hi=hi, heads=heads, kv_heads=kv, head_dim=dim, dtype=dtype, page=page,
                 len_lo=len_lo, len_hi=len_hi, evicted=evicted, frame=frame)


def _evict(name, n_seq, len_lo, len_hi, *, kv, page, keep, first, last, evicted=0):
    """Of the pages of len_lo..len_hi positions the share `keep` stays, the first and last ones in any case."""
    return _case(name, op="evict", n_seq=n_seq, heads=kv, kv_heads=kv, head_dim=64, page=page, len_lo=len_lo, len_hi=len_hi, keep=keep,
                 first=first, last=last, evicted=evicted)


def _spread(lo, hi, n, phase):
    """n whole numbers between lo and hi in no order, the first two the limits."""
    if n == 1:
        return [hi]
    return [lo, hi][:n] + [lo + int((hi - lo) * ((phase + 0.6180339887 * i) % 1.0)) for i in range(2, n)]


def _sizes(case):
    """(new tokens, held tokens) of each sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["n_seq"], 0.3)
    held = _spread(case["len_lo"], case["len_hi"], case["n_seq"], 0.7)
    if case["op"] in ("attn", "mass"):
        held = [max(a, b) for a, b in zip(held, new)]
    return new, held


def _pairs(case):
    return [case["pairs%d" % a] for a in range(case["axes"])]


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


def _row_bytes(case):
    """K or V of one token in the cache."""
    d = case["head_dim"]
    return case["kv_heads"] * {"bf16": 2 * d, "e4m3": d + 1, "e2m1": d // 2 + d // BLOCK}[case["dtype"]]


def work(case):
    new, held = _sizes(case)
    d, kv, heads = case["head_dim"], case["kv_heads"], case["heads"]
    n = sum(new)
    if case["op"] == "rope":
        return {"bytes": 2.0 * n * (heads + kv) * d * 2 + 4.0 * n * case["axes"], "flops": 6.0 * n * (heads + kv) * sum(_pairs(case))}
    if case["op"] == "store":       # rows in, codes, rows out
        return {"bytes": 2.0 * n * (2 * kv * d * 2 + _row_bytes(case)), "flops": 0.0}
    if case["op"] == "evict":
        return {"bytes": 4.0 * sum(held) * kv + 12.0 * sum(-(-m // case["page"]) for m in held), "flops": 0.0}
    seen = sum(_visible(case, a, b) for a, b in zip(new, held))
    if case["op"] == "attn":
        return {"bytes": 2.0 * 2 * n * heads * d + 2.0 * sum(held) * _row_bytes(case), "flops": 4.0 * seen * heads * d}
    return {"bytes": 2.0 * n * heads * d + 1.0 * sum(held) * (_row_bytes(case) + 8 * kv), "flops": 2.0 * seen * heads * d}


def _costs(case):
    """Bytes, flops, and about how long the plain form takes, whose scores are written and read several times."""
    w = work(case)
    new, held = _sizes(case)
    scores = max(new) * max(held) * len(new) * case["heads"] if case["op"] in ("attn", "mass") else 0
    return w["bytes"], w["flops"], w["bytes"] / 1e12 + w["flops"] / 5e13 + scores * 40.0 / 4e12


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    new, held = _sizes(case)
    n, n_seq, kv, heads, d = sum(new), case["n_seq"], case["kv_heads"], case["heads"], case["head_dim"]

    def rows(count, width):
        return torch.randn(count, width, generator=g, device=DEV, dtype=torch.bfloat16)

    def pair_of(a, b):
        """Rows of a and of b heads, as slices of one projection's output or apart."""
        if case["fused"]:
            both = rows(n, (a + b) * d)
            return both[:, :a * d].unflatten(1, (a, d)), both[:, a * d:].unflatten(1, (b, d)) if b else None
        return rows(n, a * d).unflatten(1, (a, d)), rows(n, b * d).unflatten(1, (b, d)) if b else None

    s = {"case": case, "new": new, "held": held}
    if case["op"] == "rope":
        s["q"], s["k"] = pair_of(heads, kv)
        s["pos"] = torch.stack([torch.randint(0, case["far"] if a == 0 else 40, (n,), generator=host) for a in range(case["axes"])], 1).int().to(DEV)
        s["q_out"] = torch.empty(n, heads, d, dtype=torch.bfloat16, device=DEV)
        s["k_out"] = torch.empty(n, kv, d, dtype=torch.bfloat16, device=DEV) if kv else None
        return s

    # the pool: every sequence's pages somewhere in it, some given back
    page = case["page"]
    total = [a + b for a, b in zip(new, held)] if case["op"] == "store" else held
    pages = [-(-t // page) for t in total]
    n_pages, max_pages = sum(pages) + HEADROOM, max(pages)
    where = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.full((n_seq, max_pages), -1, dtype=torch.int32)
    at = 0
    for i, c in enumerate(pages):
        table[i, :c] = where[at:at + c]
        at += c
        if case["evicted"]:      # every so many pages, but for a sequence's last one
            table[i, case["evicted"] // 2:max(c - 1, 0):case["evicted"]] = -1
    s.update(n_pages=n_pages, max_pages=max_pages, table=table.to(DEV), held_dev=torch.tensor(held, dtype=torch.int32, device=DEV))
    if case["op"] == "evict":
        # weights of unlike sizes, and pages that nobody looked at
        mass = torch.rand(n_seq, kv, max_pages * page, generator=g, device=DEV).square_()
        mass *= torch.exp(2.0 * torch.randn(n_seq, 1, max_pages, generator=g, device=DEV)).repeat_interleave(page, 2)
        s["mass"] = mass * (torch.rand(n_seq, 1, max_pages, generator=g, device=DEV) < 0.9).repeat_interleave(page, 2)
        s["keep"] = torch.tensor([int(case["keep"] * p) for p in pages], dtype=torch.int32, device=DEV)
        s["table_out"], s["freed"] = torch.empty_like(s["table"]), torch.empty_like(s["table"])
        s["n_freed"] = torch.empty(n_seq, dtype=torch.int32, device=DEV)
        return s
    s["new_off"] = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=DEV)
    shape = (n_pages, kv, page)
    gain = torch.exp(0.5 * torch.randn(kv, 1, d, generator=g, device=DEV)).to(torch.bfloat16)
    if case["op"] == "store":
        s["k"], s["v"] = pair_of(kv, kv)
        s["k"] *= gain[:, 0]
        for name in ("k", "v"):
            s["pool_" + name] = torch.zeros(*shape, d // 2, dtype=torch.uint8, device=DEV)
            s["scale_" + name] = torch.zeros(*shape, d // BLOCK, dtype=torch.uint8, device=DEV)
            s["out_" + name] = torch.empty(n, kv, d, dtype=torch.bfloat16, device=DEV)
        return s
    s["q"] = rows(n, heads * d).unflatten(1, (heads, d))
    for name in ("k", "v") if case["op"] == "attn" else ("k",):
        x = torch.randn(*shape, d, generator=g, device=DEV, dtype=torch.bfloat16)
        if name == "k":
            x *= gain
        if case["dtype"] == "bf16":
            s["pool_" + name], s["scale_" + name] = x, None
        elif case["dtype"] == "e2m1":
            s["pool_" + name], s["scale_" + name] = _quantised(x)
        else:
            _, e = torch.frexp(x.float().abs().amax(-1))
            s["pool_" + name] = (x.float() * _two_to(9 - 1 - e[..., None])).to(torch.float8_e4m3fn).view(torch.uint8)
            s["scale_" + name] = (e - 8 + 127).to(torch.uint8)
    if case["op"] == "attn":
        s["o"] = torch.empty_like(s["q"])
    else:
        # what ten such calls before gave
        s["mass_in"] = torch.rand(n_seq, kv, max_pages * page, generator=g, device=DEV) * (20.0 * (heads // kv) * max(new) / max(held))
        s["mass"] = torch.zeros(n_seq, kv, max_pages * page, device=DEV)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_2512_04939_amd import binding as B

    case = s["case"]
    op = case["op"]
    if "params" not in s:      # what a program makes once for its shapes
        if op == "rope":
            pairing = {"axis": B.ROPE_AXIS_HALVES, "head": B.ROPE_HEAD_HALVES, "adjacent": B.ROPE_ADJACENT}[case["pairing"]]
            s["params"] = B.make_rope_params(case["heads"], case["head_dim"], _pairs(case), kv_heads=case["kv_heads"], pairing=pairing,
                                             joint=int(case["joint"]), base=case["base"], inverse=int(case["inverse"]))
        else:
            s["params"] = p = B.make_cache_params(case["n_seq"], case["heads"], case["head_dim"], kv_heads=case["kv_heads"],
                                                  cache_dtype={"bf16": B.CACHE_BF16, "e4m3": B.CACHE_E4M3, "e2m1": B.CACHE_E2M1}[case["dtype"]],
                                                  page_tokens=case["page"], n_pages=s["n_pages"], max_pages=s["max_pages"],
                                                  frame_tokens=case["frame"], qk_norm=int(case["norm"]))
            s["cache"] = B.CacheBuffers(*(s.get(x) for x in ("pool_k", "pool_v", "scale_k", "scale_v")), s["table"])
            if op == "attn":
                s["ws"] = B.alloc_ws(B.litevggt_cached_attn_ws_bytes(p, s["q"].shape[0]))
            elif op == "mass":
                s["ws"] = B.alloc_ws(B.litevggt_cached_mass_ws_bytes(p, s["q"].shape[0]))
            elif op == "evict":
                s["ws"] = B.alloc_ws(B.litevggt_cache_evict_ws_bytes(p))
    p = s["params"]
    if op == "rope":
        B.litevggt_rope(p, s["pos"], s["q"], s["k"], s["q_out"], s["k_out"])
        return [s["q_out"], s["k_out"]] if case["kv_heads"] else [s["q_out"]]
    if op == "store":
        B.litevggt_cache_write(p, s["cache"], s["k"], s["v"], s["new_off"], s["held_dev"])
        B.litevggt_cache_read(p, s["cache"], s["held_dev"], s["new_off"], s["out_k"], s["out_v"])
        return [s["out_k"], s["out_v"]]
    if op == "attn":
        B.litevggt_cached_attn(p, s["cache"], s["q"], s["new_off"], s["held_dev"], s["o"], s["ws"])
        return s["o"]
    if op == "mass":
        B.litevggt_cached_mass(p, s["cache"], s["q"], s["new_off"], s["held_dev"], s["mass_in"], s["mass"], s["ws"])
        return s["mass"]
    B.litevggt_cache_evict(p, s["table"], s["held_dev"], s["mass"], s["keep"], case["first"], case["last"], s["table_out"], s["freed"],
                           s["n_freed"], s["ws"])
    return [s["table_out"], s["freed"], s["n_freed"]]


def _two_to(e):
    """2^e from its bits: pow may be an ulp off, which moves values on the border of two codes."""
    return (e.int() + 127 << 23).view(torch.float32)


def _quantised(x):
    """E2M1 codes, two to a byte, and biased exponents of rows x [..., d]."""
    f = x.float().unflatten(-1, (-1, BLOCK))
    a = f.abs().amax(-1)
    m, e = torch.frexp(a)                                    # a = m 2^e, m in [0.5, 1); 6 = 0.75 2^3
    e = torch.where(a > 0, e - 3 + (m > 0.75).int(), 0).clamp(min=-126)
    z = f * _two_to(-e[..., None])
    size = z.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    twice = (torch.round(size / step) * step * 2).to(torch.int32)      # 0 1 2 3 4 6 8 12
    code = torch.where(twice <= 4, twice, torch.where(twice == 6, 5, torch.where(twice == 8, 6, 7))) + torch.signbit(z).int() * 8
    code = code.flatten(-2).to(torch.uint8)
    return code[..., ::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _values(case, codes, scale):
    """Rows [..., d] in 32 bits of what the cache holds."""
    if case["dtype"] == "bf16":
        return codes.float()
    if case["dtype"] == "e4m3":
        return codes.view(torch.float8_e4m3fn).float() * _two_to(scale.int()[..., None] - 127)
    values = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEV)
    x = values[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, BLOCK)) * _two_to(scale.int()[..., None] - 127)).flatten(-2)


def _rows_of(s, name, page, place):
    """Rows of the cache in 32 bits [..., kv, d], zeros where a page (-1) is not held."""
    at = page.clamp(min=0)
    x = _values(s["case"], s["pool_" + name][at, :, place], None if s["scale_" + name] is None else s["scale_" + name][at, :, place])
    return x.masked_fill_((page < 0)[..., None, None], 0.0)


def _rope_plain(s):
    case, pairs = s["case"], _pairs(s["case"])
    R = sum(pairs)
    first = [sum(pairs[:a]) for a in range(len(pairs))]
    turn = torch.cat([torch.arange(p, dtype=torch.float64, device=DEV) + (f if case["joint"] else 0) for p, f in zip(pairs, first)])
    per = torch.cat([torch.full((p,), float(R if case["joint"] else p), dtype=torch.float64, device=DEV) for p in pairs])
    axis = torch.cat([torch.full((p,), a, device=DEV) for a, p in enumerate(pairs)])
    angle = s["pos"].double()[:, axis] * torch.pow(case["base"], -turn / per)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["inverse"]:
        sin = -sin
    out = []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        f = x.float()
        if case["pairing"] == "adjacent":
            a, b = f[..., :2 * R:2], f[..., 1:2 * R:2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        elif case["pairing"] == "head":
            a, b = f[..., :R], f[..., R:2 * R]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        else:
            halves = f[..., :2 * R].split([p for p in pairs for _ in range(2)], -1)
            a, b = torch.cat(halves[::2], -1), torch.cat(halves[1::2], -1)
            low, high = (a * cos - b * sin).split(pairs, -1), (b * cos + a * sin).split(pairs, -1)
            y = torch.cat([h for both in zip(low, high) for h in both], -1)
        out.append(torch.cat((y, f[..., 2 * R:]), -1).to(torch.bfloat16))
    return out


def _new_rows(s):
    """Page and place of every new token, -1 where its page is not held."""
    new = torch.tensor(s["new"], device=DEV)
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), new, output_size=s["k"].shape[0])
    pos = s["held_dev"].long()[seq] + torch.arange(s["k"].shape[0], device=DEV) - s["new_off"].long()[seq]
    return s["table"][seq, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _store_plain(s):
    page, place = _new_rows(s)
    held = (page >= 0).nonzero().squeeze(1)
    for name in ("k", "v"):
        code, e = _quantised(s[name])
        s["pool_" + name][page[held], :, place[held]] = code[held]
        s["scale_" + name][page[held], :, place[held]] = e[held]
    return [_rows_of(s, name, page, place).to(torch.bfloat16) for name in ("k", "v")]


def _weights(s, seqs):
    """Softmax weights and their divisors of some sequences at once, padded: [S, kv, group, n, m] and [S, kv, group, n, 1], the keys' page and
    place, and where the queries are."""
    case = s["case"]
    new, held = torch.tensor([s["new"][i] for i in seqs], device=DEV), torch.tensor([s["held"][i] for i in seqs], device=DEV)
    n, m = max(s["new"][i] for i in seqs), max(s["held"][i] for i in seqs)
    kv, d = case["kv_heads"], case["head_dim"]
    group = case["heads"] // kv
    i, t = torch.arange(n, device=DEV), torch.arange(m, device=DEV)
    there = i < new[:, None]
    row = torch.where(there, s["new_off"].long()[seqs[0]:seqs[-1] + 1, None] + i, 0)
    q = s["q"][row]
    if case["norm"]:
        f = q.float()
        q = (f / torch.sqrt(f.square().mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)
    q = q.float().unflatten(2, (kv, group)).permute(0, 2, 3, 1, 4).reshape(-1, group * n, d)
    page = torch.where(t < held[:, None], s["table"][seqs[0]:seqs[-1] + 1, t // case["page"]].long(), -1)
    place = (t % case["page"]).expand_as(page)
    k = _rows_of(s, "k", page, place)
    w = torch.bmm(q, k.permute(0, 2, 3, 1).reshape(-1, d, m)).mul_(1.0 / math.sqrt(d)).view(-1, kv, group, n, m)
    p = held[:, None] - new[:, None] + i
    limit = (p // case["frame"] + 1) * case["frame"] if case["frame"] else torch.full_like(p, m)
    w.masked_fill_(~((page >= 0)[:, None] & (t < limit[..., None]) & there[..., None])[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(torch.where(torch.isfinite(top), top, 0.0)).exp_()
    return w, w.sum(-1, keepdim=True), page, place, there


def _batches(s):
    """Runs of sequences whose padded scores and rows fit in memory beside the state."""
    case, runs = s["case"], [[]]
    for i in range(len(s["new"])):
        run = runs[-1] + [i]
        n, m = max(s["new"][j] for j in run), max(s["held"][j] for j in run)
        if runs[-1] and len(run) * m * (n * case["heads"] + 2 * case["kv_heads"] * case["head_dim"]) > 5e9:
            runs.append([i])
        else:
            runs[-1] = run
    return runs


def _attn_plain(s):
    case, out = s["case"], torch.zeros_like(s["q"])
    kv, d = case["kv_heads"], case["head_dim"]
    for seqs in _batches(s):
        w, total, page, place, there = _weights(s, seqs)
        v = _rows_of(s, "v", page, place).transpose(1, 2).reshape(-1, page.shape[1], d)
        o = torch.bmm(w.flatten(0, 1).flatten(1, 2), v).view(len(seqs), kv, -1, there.shape[1], d)
        o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).flatten(2, 3)
        lo = int(sum(s["new"][:seqs[0]]))
        out[lo:lo + sum(s["new"][i] for i in seqs)] = o[there].to(torch.bfloat16)
    return out


def _mass_plain(s):
    out = s["mass"].clone()
    for seqs in _batches(s):
        w, total, page, _, _ = _weights(s, seqs)
        drawn = w.mul_(torch.where(total > 0, 1.0 / total, 0.0)).flatten(2, 3).sum(2)
        m, at = page.shape[1], slice(seqs[0], seqs[-1] + 1)
        now = torch.where((page >= 0)[:, None], s["mass_in"][at, :, :m] + drawn, 0.0)
        inside = torch.arange(m, device=DEV) < s["held_dev"][at, None]
        out[at, :, :m] = torch.where(inside[:, None], now, out[at, :, :m])
    return out


def _evict_plain(s):
    case, table, columns = s["case"], s["table"], torch.arange(s["max_pages"], device=DEV)
    length = s["held_dev"].long()
    used = (length + case["page"] - 1) // case["page"]
    inside = torch.arange(s["mass"].shape[-1], device=DEV) < length[:, None]
    drawn = torch.where(inside, s["mass"].sum(1, dtype=torch.float64), 0.0).view(*table.shape, -1).sum(-1)
    held = (table >= 0) & (columns < used[:, None])
    open_ = held & (columns >= case["first"]) & (columns < used[:, None] - case["last"])
    count = torch.minimum(held.sum(1) - s["keep"].clamp(min=0), open_.sum(1)).clamp(min=0)
    order = torch.where(open_, drawn, math.inf).sort(dim=1, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, columns.expand_as(order))
    gone = open_ & (rank < count[:, None])
    freed = torch.full((table.shape[0], table.shape[1] + 1), -1, dtype=torch.int32, device=DEV)
    freed.scatter_(1, torch.where(gone, gone.cumsum(1) - 1, table.shape[1]), torch.where(gone, table, -1))
    return [torch.where(gone, -1, table), freed[:, :-1].contiguous(), count.int()]


_PLAIN = {"rope": _rope_plain, "store": _store_plain, "attn": _attn_plain, "mass": _mass_plain, "evict": _evict_plain}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _rope_exact, "store": _store_exact, "attn": _attn_exact, "mass": _attn_exact, "evict": _evict_exact}[case["op"]](s)


def _rope_exact(s):
    """A pair of channels as a complex number, times e^(i angle)."""
    case, pairs = s["case"], _pairs(s["case"])
    R, out = sum(pairs), []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        y = x.double()
        for a, p in enumerate(pairs):
            i0 = sum(pairs[:a])
            for j in range(p):
                f = case["base"] ** -((i0 + j) / R if case["joint"] else j / p)
                c1, c2 = {"adjacent": (2 * (i0 + j), 2 * (i0 + j) + 1), "head": (i0 + j, R + i0 + j), "axis": (2 * i0 + j, 2 * i0 + p + j)}[case["pairing"]]
                t = s["pos"][:, a].double() * (-f if case["inverse"] else f)
                z = torch.complex(x[..., c1].double(), x[..., c2].double()) * torch.polar(torch.ones_like(t), t)[:, None]
                y[..., c1], y[..., c2] = z.real, z.imag
        out.append(y)
    return out


def _nearest(x):
    """What rows x [..., d] (64 bits) are as E2M1 codes times a power of two for each block."""
    b = x.unflatten(-1, (-1, BLOCK))
    a = b.abs().amax(-1, keepdim=True)
    power = lambda e: (e.long() + 1023 << 52).view(torch.float64)                  # noqa: E731
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / MOST))
    e = e + (a > MOST * power(e)).double() - (a <= MOST * power(e - 1)).double()
    e = torch.where(a > 0, e, 0.0).clamp(min=-126)
    values = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    middle = (values[1:] + values[:-1]) / 2
    z = b / power(e)
    i = torch.searchsorted(middle, z.abs().contiguous())                            # middles below
    tie = z.abs() == middle[i.clamp(max=6)]
    i = i + (tie & (i < 7) & (i % 2 == 1)).long()
    return (torch.sign(z) * values[i] * power(e)).flatten(-2)


def _store_exact(s):
    out, page = [], s["case"]["page"]
    ends = torch.tensor(s["new"]).cumsum(0).tolist()
    for name in ("k", "v"):
        x = _nearest(s[name].double())
        for i, (c, h) in enumerate(zip(s["new"], s["held"])):
            there = s["table"][i].repeat_interleave(page)[h:h + c] >= 0
            x[ends[i] - c:ends[i]][~there] = 0.0
        out.append(x)
    return out


def _exact_rows(s, name, i, count):
    """The first `count` positions of sequence i, a page at a time, and which of them are held."""
    page, kind = s["case"]["page"], s["case"]["dtype"]
    ids = s["table"][i, :-(-count // page)].long()
    x = s["pool_" + name][ids.clamp(min=0)].transpose(1, 2)                          # [pages, places, kv, ..]
    if kind == "bf16":
        x = x.double()
    else:
        power = (s["scale_" + name][ids.clamp(min=0)].transpose(1, 2).long() + (1023 - 127) << 52).view(torch.float64)
        if kind == "e4m3":
            x = x.contiguous().view(torch.float8_e4m3fn).double() * power[..., None]
        else:
            size = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
            code = torch.empty(*x.shape[:-1], 2 * x.shape[-1], dtype=torch.long, device=DEV)
            code[..., 0::2], code[..., 1::2] = x % 16, x // 16
            x = size[code % 8] * (1 - 2 * (code // 8)) * power.repeat_interleave(BLOCK, -1)
    there = (ids >= 0).repeat_interleave(page)[:count]
    return x.reshape(-1, *x.shape[2:])[:count] * there[:, None, None], there


def _attn_exact(s):
    case = s["case"]
    n, heads, d = s["q"].shape
    if sum(a * b for a, b in zip(s["new"], s["held"])) * heads * d > 3e12:
        return None
    group = heads // case["kv_heads"]
    mass = case["op"] == "mass"
    out = s["mass"].double() if mass else torch.zeros(n, heads, d, dtype=torch.float64, device=DEV)
    start = 0
    for i, (c, m) in enumerate(zip(s["new"], s["held"])):
        q = s["q"][start:start + c].double()
        if case["norm"]:
            q = (q / (q.square().mean(-1, keepdim=True) + EPS).sqrt()).to(torch.bfloat16).double()
        k, there = _exact_rows(s, "k", i, m)
        v = None if mass else _exact_rows(s, "v", i, m)[0]
        t = torch.arange(m, device=DEV)
        limit = torch.full((c,), m, device=DEV)
        if case["frame"]:
            limit = (torch.arange(m - c, m, device=DEV) // case["frame"] + 1) * case["frame"]
        if mass:
            out[i, :, :m] = torch.where(there, s["mass_in"][i, :, :m].double(), 0.0)
        for b in range(0, c, 512):
            shut = ~(there & (t < limit[b:b + 512, None]))
            for h in range(heads):
                z = q[b:b + 512, h] @ k[:, h // group].t().contiguous() / math.sqrt(d)
                z[shut] = -math.inf
                best = z.max(1, keepdim=True).values
                w = torch.exp(z - torch.where(best == -math.inf, 0.0, best))
                total = w.sum(1, keepdim=True)
                w /= torch.where(total == 0, 1.0, total)
                if mass:
                    out[i, h // group, :m] += w.sum(0)
                else:
                    out[start + b:start + b + w.shape[0], h] = w @ v[:, h // group].contiguous()
        start += c
    return out


def _evict_exact(s):
    """Sequence by sequence, sorted on the host."""
    case, page = s["case"], s["case"]["page"]
    table, freed = s["table"].cpu().clone(), torch.full_like(s["table"], -1).cpu()
    count, keep = torch.zeros(len(s["held"]), dtype=torch.int32), s["keep"].tolist()
    for i, m in enumerate(s["held"]):
        used = -(-m // page)
        drawn = torch.zeros(used * page, dtype=torch.float64)
        drawn[:m] = s["mass"][i, :, :m].double().sum(0).cpu()
        drawn = drawn.view(used, page).sum(1).tolist()
        ids = table[i].tolist()
        held = [j for j in range(used) if ids[j] >= 0]
        free = sorted((j for j in held if case["first"] <= j < used - case["last"]), key=lambda j: (drawn[j], j))
        gone = sorted(free[:max(0, len(held) - max(keep[i], 0))])
        freed[i, :len(gone)] = torch.tensor([ids[j] for j in gone], dtype=torch.int32)
        table[i, gone] = -1
        count[i] = len(gone)
    return [table.to(DEV), freed.to(DEV), count.to(DEV)]
