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
