"""Refusals of the entry points for rotary positions, the E2M1 cache, drawn weight and eviction: host code, no GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2512_04939_amd import binding as B

OK, NULL, SHAPE, PARAM, WORKSPACE, DTYPE = 0, -1, -2, -3, -4, -5
P = 1 << 20      # stands for a device pointer: nothing is launched in these calls


def params(**kw):
    args = dict(n_seq=2, heads=4, head_dim=64, kv_heads=2, page_tokens=16, n_pages=8, max_pages=4, cache_dtype=B.CACHE_E2M1)
    args.update(kw)
    return B.make_cache_params(args.pop("n_seq"), args.pop("heads"), args.pop("head_dim"), **args)


def cache(**kw):
    return B.Cache(**{**dict(k=P, v=P, k_scale=P, v_scale=P, page_table=P), **kw})


def mass(p=None, c=None, n=5, q=P, qs=256, off=P, kv_len=P, had=P, out=P, ws=P, ws_bytes=1 << 40):
    p, c = p or params(), c or cache()
    return B.lib().litevggt_cached_mass(C.byref(p), C.byref(c), n, q, qs, off, kv_len, had, out, ws, ws_bytes, None)


def evict(p=None, table=P, kv_len=P, m=P, keep=P, first=0, last=0, out=P, freed=2 * P, count=P, ws=P, ws_bytes=1 << 40):
    p = p or params()
    return B.lib().litevggt_cache_evict(C.byref(p), table, kv_len, m, keep, first, last, out, freed, count, ws, ws_bytes, None)


def rope_params(**kw):
    args = dict(heads=4, head_dim=64, pairs=(16, 16), kv_heads=2)
    args.update(kw)
    return B.make_rope_params(args.pop("heads"), args.pop("head_dim"), args.pop("pairs"), **args)


def rope(p=None, n=5, pos=P, q=P, qs=256, k=P, ks=128, qo=P, qos=256, ko=P, kos=128):
    p = p or rope_params()
    return B.lib().litevggt_rope(C.byref(p), n, pos, q, qs, k, ks, qo, qos, ko, kos, None)


def test_e2m1_needs_scales():
    p = params()
    L = B.lib()
    for name in ("k_scale", "v_scale", "k", "v", "page_table"):
        c = cache(**{name: None})
        assert L.litevggt_cache_write(C.byref(p), C.byref(c), 5, P, 128, P, 128, P, P, None) == NULL
        assert L.litevggt_cache_read(C.byref(p), C.byref(c), P, P, 5, P, 128, P, 128, None) == NULL
        assert L.litevggt_cached_attn(C.byref(p), C.byref(c), 5, P, 256, P, P, P, 256, P, 1 << 40, None) == NULL
    for name in ("k_scale", "v_scale"):
        c = cache(**{name: P + 2})
        assert L.litevggt_cached_attn(C.byref(p), C.byref(c), 5, P, 256, P, P, P, 256, P, 1 << 40, None) == SHAPE
    for bad in (2, 3, 5, -1):
        assert mass(params(cache_dtype=bad)) == evict(params(cache_dtype=bad)) == DTYPE


@pytest.mark.parametrize("kw,code", [(dict(n_seq=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(head_dim=96), SHAPE), (dict(page_tokens=24), SHAPE),
                                     (dict(max_pages=0), SHAPE), (dict(frame_tokens=-1), PARAM), (dict(softmax_scale=math.nan), PARAM)], ids=str)
def test_cache_params_are_checked(kw, code):
    p = params(**kw)
    assert mass(p) == evict(p) == code
    assert B.litevggt_cached_mass_ws_bytes(p, 5) == B.litevggt_cache_evict_ws_bytes(p) == 0


def test_mass_arguments():
    for name in ("q", "off", "kv_len", "out"):
        assert mass(**{name: None}) == NULL, name
    for name in ("k", "k_scale", "page_table"):
        assert mass(c=cache(**{name: None})) == NULL, name
    assert mass(q=P + 8) == mass(out=P + 4) == mass(had=P + 8) == mass(c=cache(k=P + 4)) == SHAPE
    assert mass(qs=248) == mass(qs=260) == mass(n=-1) == mass(n=1 << 24) == SHAPE
    need = B.litevggt_cached_mass_ws_bytes(params(), 5)
    assert need > 0 and mass(ws=None) == mass(ws=P + 8) == mass(ws_bytes=need - 1) == WORKSPACE
    assert B.lib().litevggt_cached_mass(None, C.byref(cache()), 5, P, 256, P, P, P, P, P, 1 << 40, None) == NULL
    assert B.lib().litevggt_cached_mass(C.byref(params()), None, 5, P, 256, P, P, P, P, P, 1 << 40, None) == NULL


@pytest.mark.parametrize("n_seq,heads,kv,dim", [(1, 16, 16, 64), (1, 12, 1, 128), (7, 16, 4, 64), (300, 8, 2, 128), (65535, 4, 4, 64), (1, 1024, 1, 64)])
def test_scratch_for_more_tokens_serves_fewer(n_seq, heads, kv, dim):
    for columns in (1, 100, 1 << 20):
        p = params(n_seq=n_seq, heads=heads, kv_heads=kv, head_dim=dim, max_pages=columns)
        most = (1 << 26) // heads - 1
        sizes = [B.litevggt_cached_mass_ws_bytes(p, n) for n in sorted({min(most, int(1.3 ** j)) for j in range(64)})]
        assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))


def test_evict_arguments():
    for name in ("table", "kv_len", "m", "keep", "out", "freed", "count"):
        assert evict(**{name: None}) == NULL, name
    assert evict(first=-1) == evict(last=-1) == PARAM
    assert evict(m=P + 4) == evict(freed=P) == SHAPE
    need = B.litevggt_cache_evict_ws_bytes(params())
    assert need > 0 and evict(ws=None) == evict(ws=P + 8) == evict(ws_bytes=need - 1) == WORKSPACE


def test_rope_arguments():
    for name in ("pos", "q", "k", "qo", "ko"):
        assert rope(**{name: None}) == NULL, name
    assert rope(n=0, pos=None, q=None, k=None, qo=None, ko=None) == OK
    for kw, code in ((dict(heads=0), SHAPE), (dict(heads=1025), SHAPE), (dict(kv_heads=-1), SHAPE), (dict(head_dim=96), SHAPE), (dict(pairs=(0, 16)), SHAPE),
                     (dict(pairs=(16, 17)), SHAPE), (dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1)), SHAPE), (dict(pairing=3), PARAM), (dict(base=0.0), PARAM),
                     (dict(base=-1.0), PARAM), (dict(base=math.inf), PARAM), (dict(base=math.nan), PARAM), (dict(freq=[math.nan] * 32), PARAM),
                     (dict(freq=[2e6] * 32), PARAM)):
        assert rope(rope_params(**kw)) == code, kw
    five = rope_params()
    five.axes = 5
    assert rope(five) == SHAPE
    assert rope(q=P + 8) == rope(ko=P + 2) == rope(qs=248) == rope(kos=120) == rope(ks=132) == rope(n=-1) == rope(n=1 << 24) == SHAPE
    assert B.lib().litevggt_rope(None, 5, P, P, 256, P, 128, P, 256, P, 128, None) == NULL


def test_binding_refuses_what_does_not_fit():
    with pytest.raises(B.LiteVGGTError):
        rope_params(pairs=())
    with pytest.raises(B.LiteVGGTError):
        rope_params(pairs=(1, 2, 3, 4, 5))
    with pytest.raises(B.LiteVGGTError):
        rope_params(freq=[1.0] * 31)
    q, k, pos = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 2, dtype=torch.int32)
    for bad in ((pos.long(), q, k, q, k), (pos[:4], q, k, q, k), (pos, q.float(), k, q, k), (pos, q, k[:4], q, k), (pos, q, q, q, k), (pos, q, k, q[:4], k),
                (pos, q, None, q, None)):
        with pytest.raises(B.LiteVGGTError):
            B.litevggt_rope(rope_params(), *bad)
    p = params()
    c = B.alloc_cache(p, "cpu")
    assert c.k.shape == (8, 2, 16, 32) and c.k_scale.shape == (8, 2, 16, 2) and c.k.dtype == torch.uint8
    m, off, lens = B.alloc_mass(p, "cpu"), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    assert m.shape == (2, 2, 64) and not m.any()
    for bad in (m.double(), m[:1], m[..., :63], m.flatten(), m.transpose(0, 1)[:, :1]):
        with pytest.raises(B.LiteVGGTError, match="fp32"):
            B.litevggt_cached_mass(p, c, q, off, lens, None, bad, None)
        with pytest.raises(B.LiteVGGTError, match="fp32"):
            B.litevggt_cache_evict(p, c.page_table, lens, bad, lens, 0, 0, c.page_table, c.page_table.clone(), lens, None)
    for name in ("k", "v", "k_scale", "v_scale"):
        x = getattr(c, name)
        for bad in (x.float(), x[:7], x[..., :1], x.view(torch.float8_e4m3fn)):
            with pytest.raises(B.LiteVGGTError, match="wanted"):
                B.CacheBuffers(**{**c.__dict__, name: bad}).struct(p)
    t = c.page_table
    for bad in (t.long(), t[:1], t[:, :3]):
        with pytest.raises(B.LiteVGGTError):
            B.litevggt_cache_evict(p, bad, lens, m, lens, 0, 0, t, t.clone(), lens, None)


def test_a_base_may_not_give_frequencies_that_are_refused_by_themselves():
    """At most 1e6 radians a position, as for the caller's own: the last pair of 16 has base^(-15/16)."""
    for base, rc in ((1e-30, PARAM), (1e-7, PARAM), (1e-6, OK), (0.5, OK), (100.0, OK)):
        assert rope(rope_params(base=base), n=0) == rc, base
        assert rope(rope_params(base=base, joint=1), n=0) == rc, base
