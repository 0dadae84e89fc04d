"""What the paged cache's C entry points refuse before they touch a device
(no GPU needed)."""
import ctypes

import pytest

from paper_2607_22578_gb300 import _lib

A = 1 << 20                                            # an aligned address that nothing reads


def status(fn, *args):
    return getattr(_lib.load(), fn)(*args)


def message():
    return _lib.load().hs_last_error().decode()


def tables(have=A, fresh=A, n=4, n_dev=None, bt=16, table=A, width=8, pool=A, n_blocks=64,
           cursor=A, after=2 * A, starts=A, lens=A, slots=A, T=9):
    return status("hs_kv_tables", have, fresh, n, n_dev, bt, table, width, pool, n_blocks, cursor,
                  after, starts, lens, slots, T, None)


@pytest.mark.parametrize("bad,what", [
    (dict(n=-1), "n_req"), (dict(n_dev=A + 2), "n_req_dev"), (dict(n_blocks=0), "n_blocks"),
    (dict(n_blocks=1 << 28), "n_blocks"), (dict(width=0), "table_width"),
    (dict(width=1 << 27), "table_width"), (dict(T=-1), "max_tokens"), (dict(T=1 << 31), "max_tokens"),
    (dict(cursor=None), "cursor"), (dict(after=None), "cursor"), (dict(after=A), "cursor"),
    (dict(pool=None), "pool"), (dict(have=None), "have"), (dict(fresh=None), "fresh"),
    (dict(table=None), "table"), (dict(lens=None), "lens"), (dict(slots=None), "slots_out"),
    (dict(cursor=A + 4), "misaligned"), (dict(slots=A + 1), "misaligned"),
])
def test_tables_refuses(bad, what):
    assert tables(**bad) == _lib.HS_ERR_INVALID_ARG and what in message()


def test_what_there_is_no_kernel_for():
    assert tables(bt=24) == _lib.HS_ERR_UNSUPPORTED and "block_tokens" in message()
    assert tables(bt=0) == _lib.HS_ERR_UNSUPPORTED
    assert tables(n=_lib.HS_KV_MAX_REQUESTS + 1) == _lib.HS_ERR_UNSUPPORTED
    assert append(cache(bt=8)) == _lib.HS_ERR_UNSUPPORTED
    assert append(cache(d=80)) == _lib.HS_ERR_UNSUPPORTED and "dim" in message()


@pytest.mark.parametrize("bad", [dict(lens=None), dict(table=None), dict(pool=None), dict(after=A),
                                 dict(cursor=None), dict(n=-3), dict(pool=A + 2)])
def test_release_refuses(bad):
    a = dict(lens=A, n=4, n_dev=None, bt=16, table=A, width=8, pool=A, n_blocks=64, cursor=A,
             after=2 * A)
    a.update(bad)
    assert status("hs_kv_release", *a.values(), None) == _lib.HS_ERR_INVALID_ARG


def cache(k=A, v=A, ks=A, vs=A, n=64, H=2, bt=16, d=128, fmt=0):
    return _lib._KvCacheStruct(k, v, ks, vs, n, H, bt, d, fmt)


def append(c, k=A, v=A, dtype=0, T=3, slots=A):
    return status("hs_kv_append", None if c is None else ctypes.addressof(c), k, v, dtype, T, 256,
                  128, slots, None)


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(ks=None), dict(vs=None),
                                 dict(k=A + 8), dict(vs=A + 2), dict(n=0), dict(n=1 << 27),
                                 dict(H=0), dict(H=1 << 16), dict(fmt=2), dict(fmt=-1)])
def test_a_cache_that_is_none(bad):
    assert append(cache(**bad)) == _lib.HS_ERR_INVALID_ARG and message()


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(slots=None), dict(T=-1),
                                 dict(T=1 << 31), dict(dtype=2), dict(k=A + 1), dict(slots=A + 2)])
def test_append_refuses(bad):
    assert append(cache(), **bad) == _lib.HS_ERR_INVALID_ARG and message()


def attend(c=None, q=A, dtype=0, T=4, heads=8, lens=A, starts=A, n=4, n_dev=None, max_q=1, table=A,
           width=8, scale=1.0, causal=1, window=0, out=A, lse=A, ws=A, size=1 << 30):
    c = cache() if c is None else c
    return status("hs_kv_attend", ctypes.addressof(c), q, dtype, T, heads, heads * 128, 128, lens,
                  starts, n, n_dev, max_q, table, width, scale, causal, window, out, lse, ws, size,
                  None)


@pytest.mark.parametrize("bad,what", [
    (dict(heads=0), "n_heads"), (dict(heads=7), "n_heads"), (dict(T=-1), "n_tokens"),
    (dict(max_q=-1), "max_q"), (dict(max_q=1 << 30), "max_q"), (dict(T=1 << 29), "n_tokens"),
    (dict(starts=None, T=3), "starts"), (dict(width=0), "table_width"),
    (dict(width=(1 << 27) - 1), "table_width"), (dict(window=-1), "window"),
    (dict(window=3, causal=0), "window"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(dtype=5), "dtype"), (dict(q=None), "NULL"), (dict(lens=None), "NULL"),
    (dict(table=None), "NULL"), (dict(out=None), "NULL"), (dict(q=A + 1), "misaligned"),
    (dict(out=A + 8), "misaligned"), (dict(lse=A + 2), "misaligned"), (dict(n=-1), "n_req"),
])
def test_attend_refuses(bad, what):
    assert attend(**bad) == _lib.HS_ERR_INVALID_ARG and what in message()


def test_attend_workspace():
    for ws, size in ((None, 1 << 30), (A + 16, 1 << 30), (A, 1024)):
        assert attend(ws=ws, size=size) == _lib.HS_ERR_WORKSPACE
    need = _lib.load().hs_kv_attend_workspace
    assert need(8, 2, 128, 1) > 0
    for bad in ((0, 2, 128, 1), (8, 3, 128, 1), (8, 2, 96, 1), (8, 2, 128, -1)):
        assert need(*bad) == 0


def test_nothing_to_do():
    for none in (dict(n=0), dict(T=0, max_q=0), dict(max_q=0)):
        assert attend(q=None, lens=None, table=None, out=None, ws=None, **none) == _lib.HS_OK
    assert append(cache(), T=0, k=None, v=None, slots=None) == _lib.HS_OK
    assert append(None) == _lib.HS_ERR_INVALID_ARG and "cache" in message()
