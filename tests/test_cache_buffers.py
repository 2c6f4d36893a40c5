"""What the binding lets through as a cache, and from which device: the kernels check page numbers and lengths against the parameters, so the
tensors have to be what the parameters say.  Calls of no tokens: nothing is launched."""
import dataclasses

import pytest
import torch

from paper_2512_04939_amd import binding as B


class Device:
    """Stands for torch's: -1 is where CPU tensors are."""
    def __init__(self, number):
        self.number = number

    def _cuda_getDevice(self):
        return self.number

    def _cuda_getCurrentRawStream(self, number):
        return 0


@pytest.fixture(autouse=True)
def on_the_cpu(monkeypatch):
    monkeypatch.setattr(B, "_torch_c", lambda: Device(-1))


def params(e4m3, **kw):
    return B.make_cache_params(2, 4, 64, **{**dict(kv_heads=2, page_tokens=16, n_pages=8, max_pages=4, cache_dtype=int(e4m3)), **kw})


OFF, ONE = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)


def calls(p, c):
    yield lambda: B.litevggt_cache_write(p, c, None, None, OFF, ONE)
    yield lambda: B.litevggt_cache_read(p, c, ONE, OFF, None, None)
    yield lambda: B.litevggt_cached_attn(p, c, None, OFF, ONE, None, None)


def accepted(p, c):
    for call in calls(p, c):
        call()


def refused(p, c, match):
    for call in calls(p, c):
        with pytest.raises(B.LiteVGGTError, match=match):
            call()


@pytest.mark.parametrize("e4m3", [False, True])
def test_caches_that_are_what_the_parameters_say(e4m3):
    p = params(e4m3)
    c = B.alloc_cache(p, "cpu")
    accepted(p, c)
    # more pages in the pool, more sequences in the table, the same values in a row
    accepted(params(e4m3, n_pages=7), c)
    accepted(p, dataclasses.replace(c, page_table=torch.zeros(5, 4, dtype=torch.int32)))
    accepted(p, dataclasses.replace(c, k=c.k.flatten(), v=c.v.flatten(), page_table=c.page_table.flatten()))
    if e4m3:
        accepted(p, dataclasses.replace(c, k=c.k.view(torch.float8_e4m3fn), v=c.v.view(torch.float8_e4m3fn)))
    else:      # a bf16 cache has no scales; what stands there is not looked at
        accepted(p, dataclasses.replace(c, k_scale=torch.zeros(1), v_scale=None))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("name", ["k", "v"])
def test_pools_of_another_type_size_or_order(e4m3, name):
    p = params(e4m3)
    c = B.alloc_cache(p, "cpu")
    x = getattr(c, name)
    other = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16 if e4m3 else torch.uint8)
    for bad in (other, x.float(), x[:7], x[..., :32], x[:, :1], x.flatten()[:-1], torch.zeros(1, dtype=x.dtype), x.transpose(1, 2),
                x.transpose(1, 2).contiguous(), torch.cat([x, x], 3)[..., :64], x.reshape(8, 2, 32, 32)):
        refused(p, dataclasses.replace(c, **{name: bad}), f"^{name} of the cache: 8 x 2 x 16 x 64 ")
    refused(params(e4m3, n_pages=9), c, "^k of the cache: 9 x")
    refused(p, dataclasses.replace(c, **{name: None}), "failed")


@pytest.mark.parametrize("name", ["k_scale", "v_scale"])
def test_scales_of_another_type_size_or_order(name):
    p = params(True)
    c = B.alloc_cache(p, "cpu")
    x = getattr(c, name)
    for bad in (x.int(), x.float(), x[:7], x[..., :8], x.transpose(0, 1), x.flatten()[1:], x.transpose(1, 2).contiguous()):
        refused(p, dataclasses.replace(c, **{name: bad}), f"^{name}: 8 x 2 x 16 ")
    refused(p, dataclasses.replace(c, **{name: None}), "failed")


def test_page_tables_of_another_type_size_or_order():
    p = params(False)
    c = B.alloc_cache(p, "cpu")
    t = c.page_table
    for bad in (t.long(), t.float(), t[:1], t[:, :3], t.flatten()[1:], torch.zeros(4, 2, dtype=torch.int32).t(), torch.zeros(4, 2, dtype=torch.int32),
                torch.zeros(2, 5, dtype=torch.int32), torch.zeros(2, 8, dtype=torch.int32)[:, ::2]):
        refused(p, dataclasses.replace(c, page_table=bad), "^page_table: 2 x 4 ")
    refused(p, dataclasses.replace(c, page_table=None), "failed")


class Elsewhere(torch.Tensor):
    """On a second GPU, as far as the binding can see"""
    def get_device(self):
        return 1


class NothingIsCalled:
    def __getattr__(self, name):
        return lambda *args: pytest.fail(f"{name} was called")


@pytest.mark.parametrize("e4m3", [False, True])
def test_tensors_of_another_device(e4m3, monkeypatch):
    p = params(e4m3)
    c = B.alloc_cache(p, "cpu")
    x = B.make_cross_params(2, 4, 64, kv_heads=2)
    k, q = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    ws = torch.zeros(600, dtype=torch.uint8)
    every = [(B.litevggt_cache_write, [p, c, k, k, OFF, ONE]), (B.litevggt_cache_read, [p, c, ONE, OFF, k, k]),
             (B.litevggt_cached_attn, [p, c, q, OFF, ONE, q, ws]), (B.litevggt_cross_attn, [x, q, OFF, k, k, ONE, ONE, q, ws])]
    monkeypatch.setattr(B, "lib", NothingIsCalled)
    for function, args in every:      # one of the arguments, each of them
        places = [(i, lambda a: a.as_subclass(Elsewhere)) for i, a in enumerate(args) if torch.is_tensor(a)]
        for name in ("k", "v", "page_table") + (("k_scale", "v_scale") if e4m3 else ()):
            places += [(1, lambda a, name=name: dataclasses.replace(a, **{name: getattr(a, name).as_subclass(Elsewhere)}))] if c is args[1] else []
        for i, moved in places:
            with pytest.raises(B.LiteVGGTError, match="current device, cuda:-1, wanted, got one "):
                function(*[moved(a) if j == i else a for j, a in enumerate(args)])
    monkeypatch.setattr(B, "_torch_c", lambda: Device(0))
    for function, args in every:      # all of them on the CPU
        with pytest.raises(B.LiteVGGTError, match="current device, cuda:0, wanted, got one on cpu"):
            function(*args)


@pytest.mark.parametrize("size", [0, 1, 10, 255])
def test_a_workspace_that_ends_before_its_first_aligned_byte_has_none(size):
    p = params(False, max_pages=64)
    assert B.litevggt_cached_attn_ws_bytes(p, 5) > 0
    pool = torch.zeros(1024, dtype=torch.uint8)
    start = -pool.data_ptr() % 256 + 1                     # the next aligned byte is 255 behind it
    ws = pool[start:start + size]
    assert B._ws_args(ws)[1] == 0
    c, q = B.alloc_cache(p, "cpu"), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(B.LiteVGGTError, match="workspace"):
        B.litevggt_cached_attn(p, c, q, OFF, ONE, q, ws)
