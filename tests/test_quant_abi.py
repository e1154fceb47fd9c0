"""Refusals of the calls on caches in 8 or 4 bits: all before a device is touched."""
import ctypes

import pytest
import torch

from paper_2609_27373_gb300 import wise
from test_serve_abi import NULL, ODD, OFF8, PTR, cache

E4M3, E2M1 = 3, 4
INVALID, UNSUPPORTED = wise.WISE_ERR_INVALID_ARG, wise.WISE_ERR_UNSUPPORTED


def write(c, layer=0, slots=PTR, n_new=NULL, batch=1, q_len=1, dtype=0, K=PTR, V=PTR):
    return wise.load().wise_kvq_write(ctypes.byref(c), layer, slots, n_new, batch, q_len, dtype, K, V, NULL)


def read(c, layer=0, slots=PTR, first=NULL, count=NULL, batch=1, rows=1, dtype=0, K=PTR, V=PTR):
    return wise.load().wise_kv_read(ctypes.byref(c), layer, slots, first, count, batch, rows, dtype, K, V, NULL)


def attn(c, layer=0, sh=(1, 1, 2, 0, 0.0), dtype=0, Q=PTR, slots=PTR, start=NULL, lens=NULL, O=PTR):
    return wise.load().wise_kvq_attn(ctypes.byref(c), layer, ctypes.byref(wise.wise_prefix_t(*sh)), dtype, Q, slots, NULL,
                                     start, lens, O, PTR, 1 << 40, NULL)


@pytest.mark.parametrize("code", [E4M3, E2M1])
@pytest.mark.parametrize("kw,want", [
    (dict(page=24), UNSUPPORTED), (dict(head_dim=80), UNSUPPORTED), (dict(n_slots=(1 << 18) + 1), UNSUPPORTED),
    (dict(max_pages=1 << 28), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(n_layers=0), INVALID),
    (dict(pool=0), INVALID), (dict(pool=0x10008), INVALID), (dict(lens=0x10002), INVALID)])
def test_a_bad_cache(code, kw, want):
    c = cache(dtype=code, **kw)
    assert [write(c), read(c), attn(c)] == [want] * 3


@pytest.mark.parametrize("call", [write, read, attn])
def test_common_arguments(call):
    c = cache(dtype=E2M1)
    assert call(c, layer=2) == INVALID and call(c, layer=-1) == INVALID
    assert call(c, slots=NULL) == INVALID and call(c, slots=ODD) == INVALID
    for dtype in (2, 3, 4, -1):
        assert call(c, dtype=dtype) == UNSUPPORTED


@pytest.mark.parametrize("call", [write, read])
def test_rows(call):
    c, length = cache(dtype=E4M3), "q_len" if call is write else "rows"
    for bad in (NULL, OFF8):
        assert call(c, K=bad) == INVALID and call(c, V=bad) == INVALID
    assert call(c, batch=-1) == INVALID and call(c, **{length: -1}) == INVALID
    assert call(c, batch=(1 << 18) + 1) == UNSUPPORTED and call(c, **{length: 1 << 30}) == UNSUPPORTED
    assert call(c, batch=0, K=NULL) == wise.WISE_OK and call(c, **{length: 0}, K=NULL) == wise.WISE_OK


def test_lists():
    c = cache(dtype=E2M1)
    assert write(c, n_new=ODD) == INVALID
    assert read(c, first=ODD) == INVALID and read(c, count=ODD) == INVALID


def test_attention_shapes():
    c = cache(dtype=E4M3)
    assert attn(c, sh=(1, 1, 3, 0, 0.0)) == UNSUPPORTED          # heads are no multiple of kv heads
    assert attn(c, sh=(1025, 1, 2, 0, 0.0)) == UNSUPPORTED
    assert attn(c, sh=(1, 129, 2, 0, 0.0)) == UNSUPPORTED
    assert attn(c, sh=(1, 1, 2, 2, 0.0)) == UNSUPPORTED          # more groups than requests
    assert attn(c, sh=(1, 1, 2, 0, -1.0)) == INVALID and attn(c, sh=(1, 1, 2, 0, float("nan"))) == INVALID
    assert attn(c, sh=(-1, 1, 2, 0, 0.0)) == INVALID
    assert attn(c, sh=(1, 1, 2, 1, 0.0), start=PTR) == INVALID   # groups without lengths
    assert attn(c, Q=NULL) == INVALID and attn(c, O=OFF8) == INVALID
    assert attn(c, sh=(0, 1, 2, 0, 0.0), Q=NULL) == wise.WISE_OK


def test_each_kind_of_cache_has_its_calls():
    lib, sh = wise.load(), wise.wise_prefix_t(1, 1, 2, 0, 0.0)
    for code in (E4M3, E2M1):
        r = ctypes.byref(cache(dtype=code))
        assert lib.wise_kv_write(r, 0, PTR, NULL, 1, 1, PTR, PTR, NULL) == UNSUPPORTED
        assert lib.wise_prefix_attn(r, 0, ctypes.byref(sh), PTR, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == UNSUPPORTED
        assert lib.wise_prefix_attn_workspace(r, ctypes.byref(sh)) == 0
        assert lib.wise_kv_workspace(r, 4) > 0
    c = cache()
    assert write(c) == UNSUPPORTED and attn(c) == UNSUPPORTED
    assert lib.wise_kvq_attn_workspace(ctypes.byref(c), ctypes.byref(sh)) == 0
    assert read(c, dtype=1) == UNSUPPORTED                       # a cache of 16 bits is read in its own type


def test_block_bytes():
    for page in (16, 32, 64, 128):
        for dim, extra in ((64, 8), (96, 14), (128, 16)):
            assert wise.kvq_block_bytes(page, dim, 4) == page * (dim + extra)
            assert wise.kvq_block_bytes(page, dim, 8) == page * (2 * dim + extra)
    for bad in ((24, 64, 4), (16, 80, 4), (16, 64, 2), (16, 64, 16)):
        with pytest.raises(ValueError):
            wise.kvq_block_bytes(*bad)


def test_cache_arguments(monkeypatch):
    monkeypatch.setattr(wise, "_check", lambda *a: None)
    size = wise.kvq_block_bytes(16, 64, 4)
    lists = [torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
    pool = torch.zeros((1, 3, 2, size), dtype=torch.uint8)
    c = wise.Cache(pool, *lists, bits=4, page=16, head_dim=64, dtype=torch.float16)
    assert (c.n_layers, c.n_pages, c.n_kv_heads, c.page, c.head_dim, c.bits, c.dtype) == (1, 3, 2, 16, 64, 4, torch.float16)
    for kw in (dict(bits=4, page=16, head_dim=64), dict(bits=4, page=32, head_dim=64, dtype=torch.float16),
               dict(bits=8, page=16, head_dim=64, dtype=torch.float16), dict(bits=5, page=16, head_dim=64, dtype=torch.float16),
               dict(bits=4, head_dim=64, dtype=torch.float16), dict(bits=4, page=16, head_dim=64, dtype=torch.float32)):
        with pytest.raises(ValueError):
            wise.Cache(pool, *lists, **kw)
    plain = torch.zeros((2, 3, 2, 16, 64), dtype=torch.bfloat16)
    assert wise.Cache(plain, *lists).bits == 16
    with pytest.raises(ValueError):
        wise.Cache(plain, *lists, page=32)


class Library:
    """Takes down which calls are made."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 64 if name.endswith("workspace") or name.endswith("bytes") else 0
        return call


def test_a_cache_makes_the_calls_of_its_kind(monkeypatch):
    """PagedCache.write, attend and read with 16 and with fewer bits; keys of another type than the cache's are refused."""
    from paper_2609_27373_gb300 import serve
    lib = Library()
    monkeypatch.setattr(wise, "load", lambda: lib)
    monkeypatch.setattr(wise, "_check", lambda *a: None)
    monkeypatch.setattr(wise, "_current_raw", lambda index: 0)
    monkeypatch.setattr(wise, "_current_device", lambda: -1)
    monkeypatch.setattr(serve.PagedCache, "_use", lambda self, stream: 0)
    monkeypatch.setattr(serve, "_empty", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    lists = [torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
    slots = torch.zeros(1, dtype=torch.int32)
    for bits, write, attn in ((16, "wise_kv_write", "wise_prefix_attn"), (8, "wise_kvq_write", "wise_kvq_attn"),
                              (4, "wise_kvq_write", "wise_kvq_attn")):
        if bits == 16:
            c = serve.PagedCache.over(torch.zeros((2, 3, 2, 16, 64), dtype=torch.float16), *lists)
        else:
            c = serve.PagedCache.over(torch.zeros((1, 3, 2, 64), dtype=torch.uint8), *lists, bits=bits, page=16, head_dim=64,
                                      dtype=torch.float16)
        x = torch.zeros((1, 2, 1, 64), dtype=torch.float16)
        lib.calls.clear()
        c.write(0, slots, None, x, x)
        c.attend(0, x, x.clone(), slots)
        c.read(0, x, x.clone(), slots)
        assert lib.calls == [write, attn + "_workspace", attn, "wise_kv_read"]
        for call in (lambda y: c.write(0, slots, None, y, y), lambda y: c.attend(0, y, y, slots), lambda y: c.read(0, y, y, slots)):
            for bad in (x.bfloat16(), torch.zeros((1, 2, 1, 128), dtype=torch.float16)[..., ::2],
                        torch.zeros((1, 2, 1, 32), dtype=torch.float16)):
                with pytest.raises(ValueError):
                    call(bad)
