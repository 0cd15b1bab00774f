"""CPU test: the page calls launch kernels on the cache's memory, so a cache on another device than the current one is refused."""
import numpy as np
import pytest

from test_chunk_host import Fake, ck  # noqa: F401 (ck: a fixture)


def test_a_cache_on_another_device_is_refused(ck, monkeypatch):  # noqa: F811
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ck, "_raw_stream", lambda device: 0)
    f = Fake(ck, [100, 100], B=2, pages=(8, 4))

    class Cache:
        B, struct = 2, f.st
        k_pool = torch.zeros(1)  # not on the current device

    before = f.state()
    for call in (lambda: ck.catekv_pages_reserve(Cache, 100), lambda: ck.catekv_fork(Cache, np.array([0, 0])), lambda: ck.catekv_truncate(Cache, [1, 0]),
                 lambda: ck.catekv_pages_compact(Cache)):
        with pytest.raises(ck.CatekvError) as e:
            call()
        assert e.value.code == ck.ERR_INVALID_ARG
    assert f.state() == before


def test_reserving_by_sequence_is_refused(ck):  # noqa: F811
    import ctypes as C
    f = Fake(ck, [128, 128], B=2, pages=(3, 4))
    before = f.state()
    call = lambda *n: ck._lib.catekv_pages_reserve_each(C.byref(f.st), np.array(n, dtype=np.int32).ctypes.data_as(C.c_void_p), None)
    assert ck._lib.catekv_pages_reserve_each(C.byref(f.st), None, None) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_pages_reserve_each(None, None, None) == ck.ERR_INVALID_ARG
    assert call(-1, 0) == call(0, -1) == ck.ERR_INVALID_ARG
    assert call(0, 0) == ck.OK
    assert call(200, 1) == ck.ERR_CAPACITY            # five pages, three are there
    assert call(257, 0) == call(2 ** 31 - 1, 0) == ck.ERR_CAPACITY  # a table row of four pages
    g = Fake(ck, [128, 128], B=2)
    assert ck._lib.catekv_pages_reserve_each(C.byref(g.st), np.zeros(2, dtype=np.int32).ctypes.data_as(C.c_void_p), None) == ck.ERR_INVALID_ARG  # no pages
    assert f.state() == before
