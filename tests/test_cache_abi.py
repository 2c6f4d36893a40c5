"""Refusals of the cache's and the attentions' entry points: argument checks are host code and run without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2512_04939_amd import binding as B

OK, NULL, SHAPE, PARAM, WORKSPACE, DTYPE = 0, -1, -2, -3, -4, -5
P = 1 << 20      # stands for a device pointer: nothing is launched in these calls


def params(**kw):
    args = dict(n_seq=2, heads=4, head_dim=64, kv_heads=2, page_tokens=16, n_pages=8, max_pages=4)
    args.update(kw)
    return B.make_cache_params(args.pop("n_seq"), args.pop("heads"), args.pop("head_dim"), **args)


def cache(**kw):
    return B.Cache(**{**dict(k=P, v=P, k_scale=P, v_scale=P, page_table=P), **kw})


def write(p=None, c=None, n=5, k=P, ks=128, v=P, vs=128, off=P, pos=P):
    p, c = p or params(), c or cache()
    return B.lib().litevggt_cache_write(C.byref(p), C.byref(c), n, k, ks, v, vs, off, pos, None)


def read(p=None, c=None, n=5, k=P, ks=128, v=P, vs=128, off=P, first=P):
    p, c = p or params(), c or cache()
    return B.lib().litevggt_cache_read(C.byref(p), C.byref(c), first, off, n, k, ks, v, vs, None)


def cached(p=None, c=None, n=5, q=P, qs=256, off=P, kv_len=P, o=P, os=256, ws=P, ws_bytes=1 << 40):
    p, c = p or params(), c or cache()
    return B.lib().litevggt_cached_attn(C.byref(p), C.byref(c), n, q, qs, off, kv_len, o, os, ws, ws_bytes, None)


def cross(p=None, n=5, q=P, qs=256, off=P, m=7, k=P, ks=128, v=P, vs=128, begin=P, end=P, o=P, os=256, ws=P, ws_bytes=1 << 40):
    p = p or B.make_cross_params(2, 4, 64, kv_heads=2)
    return B.lib().litevggt_cross_attn(C.byref(p), n, q, qs, off, m, k, ks, v, vs, begin, end, o, os, ws, ws_bytes, None)


BAD_PARAMS = [(dict(n_seq=0), SHAPE), (dict(n_seq=65536), SHAPE), (dict(heads=5), SHAPE), (dict(kv_heads=0), SHAPE),
              (dict(heads=2, kv_heads=4), SHAPE), (dict(heads=2048, kv_heads=2), SHAPE), (dict(head_dim=96), SHAPE),
              (dict(page_tokens=8), SHAPE), (dict(page_tokens=48), SHAPE), (dict(page_tokens=2048), SHAPE),
              (dict(page_tokens=-16), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE),
              (dict(page_tokens=1024, max_pages=1 << 21), SHAPE), (dict(frame_tokens=-1), PARAM),
              (dict(cache_dtype=2), DTYPE), (dict(softmax_scale=float("nan")), PARAM), (dict(softmax_scale=float("inf")), PARAM)]


@pytest.mark.parametrize("kw,code", BAD_PARAMS, ids=[str(b[0]) for b in BAD_PARAMS])
def test_cache_params_are_checked_by_every_call(kw, code):
    p = params(**kw)
    assert write(p) == read(p) == cached(p) == code
    assert B.litevggt_cached_attn_ws_bytes(p, 5) == 0


def test_null_pointers():
    L = B.lib()
    assert L.litevggt_cache_write(None, C.byref(cache()), 5, P, 128, P, 128, P, P, None) == NULL
    assert L.litevggt_cached_attn(C.byref(params()), None, 5, P, 256, P, P, P, 256, P, 1 << 40, None) == NULL
    assert L.litevggt_cross_attn(None, 5, P, 256, P, 7, P, 128, P, 128, P, P, P, 256, P, 1 << 40, None) == NULL
    for name in ("k", "v", "page_table"):
        c = cache(**{name: None})
        assert write(c=c) == read(c=c) == cached(c=c) == NULL, name
    e4m3 = params(cache_dtype=B.CACHE_E4M3)
    for name in ("k_scale", "v_scale"):
        assert write(e4m3, cache(**{name: None})) == cached(e4m3, cache(**{name: None})) == NULL
    for name in ("k", "v", "off", "pos"):
        assert write(**{name: None}) == NULL, name
    for name in ("k", "v", "off", "first"):
        assert read(**{name: None}) == NULL, name
    for name in ("q", "off", "kv_len", "o"):
        assert cached(**{name: None}) == NULL, name
    for name in ("q", "off", "k", "v", "begin", "end", "o"):
        assert cross(**{name: None}) == NULL, name


@pytest.mark.parametrize("stride", [0, 120, 127, 132, -128, (1 << 26) + 8])
def test_row_strides(stride):
    assert write(ks=stride) == write(vs=stride) == read(ks=stride) == read(vs=stride) == SHAPE
    assert cross(ks=stride) == cross(vs=stride) == SHAPE
    if stride < 256:
        assert cached(qs=stride) == cached(os=stride) == cross(qs=stride) == cross(os=stride) == SHAPE


def test_alignment_and_counts():
    assert write(k=P + 8) == read(v=P + 2) == cached(q=P + 8) == cached(o=P + 4) == cross(k=P + 8) == SHAPE
    assert write(c=cache(k=P + 8)) == SHAPE
    assert write(n=-1) == read(n=-1) == cached(n=-1) == cross(n=-1) == cross(m=-1) == SHAPE
    assert write(n=1 << 30) == read(n=1 << 30) == cached(n=1 << 29) == cross(n=1 << 29) == cross(m=1 << 30) == SHAPE


def test_nothing_to_do_is_no_error():
    assert write(n=0, k=None, v=None) == read(n=0, k=None, v=None) == OK
    assert cached(n=0, q=None, o=None, ws=None, ws_bytes=0) == OK
    assert cross(n=0, q=None, o=None, ws=None, ws_bytes=0) == cross(n=0, q=None, o=None, m=0, k=None, v=None) == OK


def test_workspace():
    p = params(max_pages=64)
    need = B.litevggt_cached_attn_ws_bytes(p, 5)
    assert need > 0
    assert cached(p, ws=None) == cached(p, ws_bytes=need - 1) == cached(p, ws=P + 128) == WORKSPACE
    x = B.make_cross_params(2, 4, 64, kv_heads=2)
    need = B.litevggt_cross_attn_ws_bytes(x, 5, 3000)
    assert need > 0
    assert cross(x, m=3000, ws=None) == cross(x, m=3000, ws_bytes=need - 1) == WORKSPACE
    xn = B.make_cross_params(2, 4, 64, kv_heads=2, qk_norm=1)
    assert B.litevggt_cross_attn_ws_bytes(xn, 5, 3000) >= need + 3000 * 2 * 64 * 2
    assert B.litevggt_cross_attn_ws_bytes(x, 0, 3000) == 0 == B.litevggt_cross_attn_ws_bytes(x, 5, -1)


def test_cross_params_are_checked():
    for kw, code in (({"kv_heads": 3}, SHAPE), ({"softmax_scale": float("nan")}, PARAM)):
        assert cross(B.make_cross_params(2, 4, 64, **kw)) == code
    for args in ((0, 4, 64), (65536, 4, 64), (2, 0, 64), (2, 4, 32), (2, 2000, 64)):
        assert cross(B.make_cross_params(*args)) == SHAPE, args


def test_binding_refuses_what_rows_cannot_be():
    p = params()
    c = B.CacheBuffers(*(torch.zeros(1) for _ in range(5)))
    good = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    for bad in (good.float(), good[..., :32], torch.zeros(5, 64, 2, dtype=torch.bfloat16).transpose(1, 2), good[0],
                torch.zeros(5, 4, 64, dtype=torch.bfloat16)[:, ::2], good.transpose(1, 2)):
        with pytest.raises(B.LiteVGGTError):
            B.litevggt_cache_write(p, c, bad, good, i, i)
        with pytest.raises(B.LiteVGGTError):
            B.litevggt_cache_read(p, c, i, i, good, bad)
    with pytest.raises(B.LiteVGGTError, match="rows"):
        B.litevggt_cache_write(p, c, good, good[:4], i, i)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(B.LiteVGGTError, match="rows"):
        B.litevggt_cached_attn(p, c, q, i, i, q[:3], None)


def test_largest_calls():
    assert write(n=1 << 24) == read(n=1 << 24) == cached(n=1 << 24) == cross(n=1 << 24) == cross(m=1 << 24) == SHAPE
    wide = params(n_seq=2, heads=16, kv_heads=16)
    assert write(wide, n=1 << 23, ks=1024, vs=1024) == cached(wide, n=1 << 23, qs=1024, os=1024) == SHAPE
    assert B.litevggt_cached_attn_ws_bytes(wide, 1 << 23) == 0
    many = params(n_seq=65535, heads=128, kv_heads=128)
    assert write(many, ks=8192, vs=8192) == cached(many, qs=8192, os=8192) == SHAPE


@pytest.mark.parametrize("n_seq,heads,kv,dim,e4m3", [(1, 16, 16, 64, False), (1, 12, 1, 128, True), (7, 16, 4, 64, True), (64, 16, 16, 64, False),
                                                     (300, 8, 2, 128, False), (4096, 16, 16, 128, True), (65535, 4, 4, 64, False)])
def test_scratch_for_more_tokens_serves_fewer(n_seq, heads, kv, dim, e4m3):
    p = params(n_seq=n_seq, heads=heads, kv_heads=kv, head_dim=dim, cache_dtype=int(e4m3), max_pages=4096)
    x = B.make_cross_params(n_seq, heads, dim, kv_heads=kv)
    group = heads // kv
    counts = sorted({max(1, c + e) for c in [32 * n_seq // group, 64 * n_seq // group] + [int(1.3 ** j) for j in range(56)] for e in (-1, 0, 1)})
    for sizes in ([B.litevggt_cached_attn_ws_bytes(p, n) for n in counts], [B.litevggt_cross_attn_ws_bytes(x, n, 100000) for n in counts]):
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))
        assert 0 < sizes[0] and sizes[-1] < 512 << 20


def test_binding_refuses_numbers_that_are_not_int32():
    p = params()
    c = B.CacheBuffers(*(torch.zeros(1) for _ in range(5)))
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    off, one = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    x = B.make_cross_params(2, 4, 64, kv_heads=2)
    for bad in (off.long(), off[:1], torch.zeros(6, dtype=torch.int32)[::2], off.float()):
        for call in (lambda a, b: B.litevggt_cache_write(p, c, k, k, a, b), lambda a, b: B.litevggt_cache_read(p, c, b, a, k, k),
                     lambda a, b: B.litevggt_cached_attn(p, c, q, a, b, q, None),
                     lambda a, b: B.litevggt_cross_attn(x, q, a, k, k, b, b, q, None)):
            with pytest.raises(B.LiteVGGTError, match="int32"):
                call(bad, one)
            with pytest.raises(B.LiteVGGTError, match="int32"):
                call(off, bad)
