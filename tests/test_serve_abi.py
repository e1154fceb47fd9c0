"""Host-side checks of the serving calls: every refusal below happens before a
device is touched, so it is tested without one."""
import ctypes

import pytest

from paper_2609_27373_gb300 import wise

NULL = ctypes.c_void_p(0)
PTR = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10002)
OFF8 = ctypes.c_void_p(0x10008)


def cache(**kw):
    d = dict(n_pages=8, page=16, n_slots=4, max_pages=4, n_layers=2, n_kv_heads=2, head_dim=64, dtype=0,
             pool=0x10000, table=0x10000, lens=0x10000, refs=0x10000)
    d.update(kw)
    return wise.wise_cache_t(*d.values())


def all_calls(c):
    """Status of every cache call on cache c, with lists that would do."""
    lib, r = wise.load(), ctypes.byref(c)
    sh = wise.wise_prefix_t(1, 1, 2, 0, 0.0)
    return [lib.wise_kv_fork(r, PTR, PTR, 1, NULL), lib.wise_kv_extend(r, PTR, PTR, 1, PTR, PTR, NULL),
            lib.wise_kv_write(r, 0, PTR, NULL, 1, 1, PTR, PTR, NULL), lib.wise_kv_drop(r, PTR, PTR, 1, NULL),
            lib.wise_kv_compact(r, PTR, PTR, PTR, NULL),
            lib.wise_prefix_attn(r, 0, ctypes.byref(sh), PTR, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL)]


@pytest.mark.parametrize("kw,code", [
    (dict(page=24), wise.WISE_ERR_UNSUPPORTED),
    (dict(page=256), wise.WISE_ERR_UNSUPPORTED),
    (dict(head_dim=80), wise.WISE_ERR_UNSUPPORTED),
    (dict(dtype=2), wise.WISE_ERR_UNSUPPORTED),
    (dict(n_slots=(1 << 18) + 1), wise.WISE_ERR_UNSUPPORTED),
    (dict(max_pages=1 << 28), wise.WISE_ERR_UNSUPPORTED),
    (dict(n_pages=1 << 30), wise.WISE_ERR_UNSUPPORTED),
    (dict(n_pages=(1 << 30) - 2, n_kv_heads=4), wise.WISE_ERR_UNSUPPORTED),
    (dict(n_pages=0), wise.WISE_ERR_INVALID_ARG),
    (dict(n_slots=-1), wise.WISE_ERR_INVALID_ARG),
    (dict(n_kv_heads=0), wise.WISE_ERR_INVALID_ARG),
    (dict(n_layers=0), wise.WISE_ERR_INVALID_ARG),
    (dict(table=0), wise.WISE_ERR_INVALID_ARG),
    (dict(lens=0x10002), wise.WISE_ERR_INVALID_ARG),
    (dict(refs=0), wise.WISE_ERR_INVALID_ARG),
])
def test_every_call_refuses_a_bad_cache(kw, code):
    assert all_calls(cache(**kw)) == [code] * 6
    assert wise.load().wise_kv_workspace(ctypes.byref(cache(**kw)), 4) == 0


def test_null_and_misaligned_arguments():
    lib = wise.load()
    c = cache()
    r, bad = ctypes.byref(c), wise.WISE_ERR_INVALID_ARG
    nopool = cache(pool=0)
    assert lib.wise_kv_compact(ctypes.byref(nopool), PTR, PTR, PTR, NULL) == bad
    assert lib.wise_kv_fork(r, NULL, PTR, 1, NULL) == bad
    assert lib.wise_kv_fork(r, PTR, ODD, 1, NULL) == bad
    assert lib.wise_kv_fork(r, PTR, PTR, -1, NULL) == bad
    assert lib.wise_kv_fork(None, PTR, PTR, 1, NULL) == bad
    assert lib.wise_kv_extend(r, PTR, PTR, 1, NULL, PTR, NULL) == bad
    assert lib.wise_kv_extend(r, PTR, PTR, 1, PTR, OFF8, NULL) == bad
    assert lib.wise_kv_write(r, 2, PTR, NULL, 1, 1, PTR, PTR, NULL) == bad      # layer past the last
    assert lib.wise_kv_write(r, -1, PTR, NULL, 1, 1, PTR, PTR, NULL) == bad
    assert lib.wise_kv_write(r, 0, PTR, NULL, 1, 1, PTR, OFF8, NULL) == bad
    assert lib.wise_kv_drop(r, PTR, NULL, 1, NULL) == bad
    assert lib.wise_kv_compact(r, NULL, PTR, PTR, NULL) == bad


def test_write_counts_rows_in_32_bits():
    lib, r = wise.load(), ctypes.byref(cache(n_kv_heads=2))
    assert lib.wise_kv_write(r, 0, PTR, NULL, 1, (1 << 29) + 1, PTR, PTR, NULL) == wise.WISE_ERR_UNSUPPORTED
    assert lib.wise_kv_write(r, 0, PTR, NULL, 1 << 10, (1 << 19) + 1, PTR, PTR, NULL) == wise.WISE_ERR_UNSUPPORTED


def test_empty_lists_do_nothing():
    lib, r = wise.load(), ctypes.byref(cache())
    assert lib.wise_kv_fork(r, NULL, NULL, 0, NULL) == 0
    assert lib.wise_kv_extend(r, NULL, NULL, 0, NULL, NULL, NULL) == 0
    assert lib.wise_kv_write(r, 0, NULL, NULL, 0, 3, NULL, NULL, NULL) == 0
    assert lib.wise_kv_write(r, 0, NULL, NULL, 3, 0, NULL, NULL, NULL) == 0
    assert lib.wise_kv_drop(r, NULL, NULL, 0, NULL) == 0
    sh = wise.wise_prefix_t(0, 1, 2, 0, 0.0)
    assert lib.wise_prefix_attn(r, 0, ctypes.byref(sh), NULL, NULL, NULL, NULL, NULL, NULL, NULL, 0, NULL) == 0
    assert lib.wise_prefix_attn_workspace(r, ctypes.byref(sh)) == 0
    assert lib.wise_verify_draft(0, 2, 10, 2, *[NULL] * 9) == 0


@pytest.mark.parametrize("sh,code", [
    ((1, 1, 3, 0, 0.0), wise.WISE_ERR_UNSUPPORTED),        # 3 heads over 2
    ((1025, 1, 2, 0, 0.0), wise.WISE_ERR_UNSUPPORTED),     # batch
    ((1, 129, 2, 0, 0.0), wise.WISE_ERR_UNSUPPORTED),      # rows of a request and kv head
    ((1, 65, 4, 0, 0.0), wise.WISE_ERR_UNSUPPORTED),
    ((2, 1, 2, 3, 0.0), wise.WISE_ERR_UNSUPPORTED),        # more groups than requests
    ((-1, 1, 2, 0, 0.0), wise.WISE_ERR_INVALID_ARG),
    ((1, -1, 2, 0, 0.0), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 0, 0, 0.0), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 2, -1, 0.0), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 2, 0, -1.0), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 2, 0, float("nan")), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 2, 0, float("inf")), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 2, 1, 0.0), wise.WISE_ERR_INVALID_ARG),        # groups without their arrays
])
def test_attention_shape_checks(sh, code):
    c = cache()
    s = wise.wise_prefix_t(*sh)
    assert wise.load().wise_prefix_attn(ctypes.byref(c), 0, ctypes.byref(s), PTR, PTR, NULL, NULL, NULL, PTR, PTR,
                                        1 << 40, NULL) == code


def test_attention_pointer_checks():
    c, s = cache(), wise.wise_prefix_t(1, 1, 2, 0, 0.0)
    call = wise.load().wise_prefix_attn
    r, sr, bad = ctypes.byref(c), ctypes.byref(s), wise.WISE_ERR_INVALID_ARG
    assert call(r, 0, sr, NULL, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad
    assert call(r, 0, sr, OFF8, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad
    assert call(r, 0, sr, PTR, NULL, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad
    assert call(r, 0, sr, PTR, PTR, ODD, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad
    assert call(r, 0, sr, PTR, PTR, NULL, NULL, NULL, OFF8, PTR, 1 << 40, NULL) == bad
    assert call(r, 2, sr, PTR, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad
    assert call(r, 0, None, PTR, PTR, NULL, NULL, NULL, PTR, PTR, 1 << 40, NULL) == bad


@pytest.mark.parametrize("args,code", [
    ((-1, 1, 10, 2, PTR, PTR), wise.WISE_ERR_INVALID_ARG),
    ((1, -1, 10, 2, PTR, PTR), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 0, 2, PTR, PTR), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 10, 3, PTR, PTR), wise.WISE_ERR_UNSUPPORTED),
    ((1, 1, (1 << 18) + 1, 2, PTR, PTR), wise.WISE_ERR_UNSUPPORTED),
    ((1, 1025, 10, 2, PTR, PTR), wise.WISE_ERR_UNSUPPORTED),
    ((1, 1, 10, 2, NULL, PTR), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 10, 2, PTR, NULL), wise.WISE_ERR_INVALID_ARG),
    ((1, 1, 10, 2, ODD, PTR), wise.WISE_ERR_INVALID_ARG),
])
def test_verification_argument_checks(args, code):
    assert wise.load().wise_verify_draft(*args, PTR, NULL, PTR, PTR, PTR, PTR, NULL) == code


def test_workspace_covers_its_lists():
    c = cache(n_pages=1000)
    lib = wise.load()
    assert lib.wise_kv_workspace(ctypes.byref(c), 0) >= 8 * 1000
    assert lib.wise_kv_workspace(ctypes.byref(c), 50) >= 4 * (1000 + 4 * 50)
