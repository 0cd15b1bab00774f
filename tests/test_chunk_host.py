"""CPU tests of the chunk and page calls: what they refuse (nothing is launched, nothing changes) and what is decided on the host."""
import ctypes as C

import numpy as np
import pytest

F = 0x10000  # stands for device memory; nothing dereferences it here


@pytest.fixture(scope="module")
def ck():
    from paper_2608_30295_b200 import build
    build.build()
    from paper_2608_30295_b200 import binding
    return binding


class Fake:
    """A cache descriptor over device memory that is not there."""

    def __init__(self, ck, lens, B=1, max_new=0, pages=None, caps=True):
        Hkv = len(lens) // B
        self.off, self.cap, total = ck.catekv_cache_layout(B, Hkv, lens, max_new)
        self.len = np.array(lens, dtype=np.int32)
        self.st = ck.CacheStruct(B, Hkv, 128, 0, total, F, F, F, F, self.off.ctypes.data, self.cap.ctypes.data, self.len.ctypes.data, None, F if caps else None)
        if pages is not None:
            n_pages, max_pages = pages
            self.table = np.full((len(lens), max_pages), -1, dtype=np.int32)
            self.seg_pages = np.zeros(len(lens), dtype=np.int32)
            self.pages = ck.PagesStruct(max_pages, n_pages, 0, 0, F, F, F, self.table.ctypes.data, self.seg_pages.ctypes.data, F if caps else None)
            self.st.pages = C.pointer(self.pages)

    def give(self, s, *pages):
        self.table[s, :len(pages)] = pages
        self.seg_pages[s] = len(pages)
        self.pages.next_free = max(self.pages.next_free, max(pages) + 1)

    def state(self):
        p = getattr(self, "pages", None)
        return ([self.off.tolist(), self.cap.tolist(), self.len.tolist()]
                + ([self.table.tolist(), self.seg_pages.tolist(), p.next_free, p.released] if p else []))


def chunk(ck, n_new, start=None, n_tokens=None, B=None):
    n = np.array(n_new, dtype=np.int32)
    s = None if start is None else np.array(start, dtype=np.int32)
    c = ck.ChunkStruct(len(n_new) if B is None else B, int(n.sum()) if n_tokens is None else n_tokens, n.ctypes.data, None if s is None else s.ctypes.data)
    c.keep = (n, s)
    return c


def append(ck, f, c, k=F, v=F, st_t=256, st_h=128):
    return ck._lib.catekv_append_chunk(C.byref(f.st), C.byref(c), k, v, st_t, st_h, None)


def attend(ck, f, c, Hq=4, q=F, st_t=512, st_h=128, scale=0.0, out=F, dt=0, lse=F, ws=F, wb=1 << 40):
    return ck._lib.catekv_chunk_attn(C.byref(f.st), C.byref(c), q, st_t, st_h, Hq, scale, out, dt, lse, ws, wb, None)


def both(ck, f, c):
    return {append(ck, f, c), attend(ck, f, c)}


def test_chunks_that_are_refused(ck):
    f = Fake(ck, [300, 300, 300, 300], B=2, max_new=100)
    before = f.state()
    bad = {ck.ERR_INVALID_ARG}
    assert both(ck, f, chunk(ck, [3])) == bad                                # another number of sequences
    assert both(ck, f, chunk(ck, [-1, 3], n_tokens=3)) == bad
    assert both(ck, f, chunk(ck, [2, 2], n_tokens=3)) == bad                 # more tokens than the axis has
    assert both(ck, f, chunk(ck, [2, 2], [0, 2], 3)) == bad
    assert both(ck, f, chunk(ck, [2, 2], [-1, 2], 9)) == bad
    assert both(ck, f, chunk(ck, [2, 2], [3, 2], 9)) == bad                  # a token of two sequences
    assert both(ck, f, chunk(ck, [4, 1], [2, 3], 9)) == bad
    assert both(ck, f, chunk(ck, [2 ** 31 - 1, 5], n_tokens=2 ** 31 - 1)) == bad
    assert ck._lib.catekv_append_chunk(C.byref(f.st), None, F, F, 256, 128, None) == ck.ERR_INVALID_ARG
    assert f.state() == before
    big = Fake(ck, [10] * 513, B=513)
    assert both(ck, big, chunk(ck, [1] * 513)) == {ck.ERR_UNSUPPORTED}
    # nothing to do: nothing is looked at, nothing launched
    assert append(ck, f, chunk(ck, [0, 0]), None, None) == ck.OK == attend(ck, f, chunk(ck, [0, 0]), q=None, out=None, ws=None)
    assert append(ck, f, chunk(ck, [0, 0], [7, 7], 7), None, None) == ck.OK
    assert f.state() == before


def test_appends_that_are_refused(ck):
    f = Fake(ck, [120, 100], max_new=0)
    before = f.state()
    assert append(ck, f, chunk(ck, [9])) == ck.ERR_CAPACITY                  # 128 rows each
    assert append(ck, f, chunk(ck, [2 ** 31 - 1])) == ck.ERR_CAPACITY
    c = chunk(ck, [8])
    for k, v, t, h, code in ((None, F, 256, 128, ck.ERR_INVALID_ARG), (F, None, 256, 128, ck.ERR_INVALID_ARG), (F + 8, F, 256, 128, ck.ERR_INVALID_ARG),
                             (F, F, 252, 128, ck.ERR_UNSUPPORTED), (F, F, 256, 130, ck.ERR_UNSUPPORTED), (F, F, 0, 128, ck.ERR_UNSUPPORTED),
                             (F, F, -256, 128, ck.ERR_UNSUPPORTED), (F, F, 256, 64, ck.ERR_UNSUPPORTED)):
        assert append(ck, f, c, k, v, t, h) == code
    assert append(ck, Fake(ck, [100], caps=False), chunk(ck, [1])) == ck.ERR_INVALID_ARG
    assert f.state() == before
    p = Fake(ck, [128, 128], pages=(4, 2))
    p.give(0, 0), p.give(1, 1)
    assert append(ck, p, chunk(ck, [65])) == ck.ERR_CAPACITY                 # the pages it has, not those it may get


def test_attention_that_is_refused(ck):
    f = Fake(ck, [300, 300], max_new=0)
    c = chunk(ck, [3])
    inv, uns = ck.ERR_INVALID_ARG, ck.ERR_UNSUPPORTED
    for kw, code in (({"Hq": 0}, inv), ({"Hq": 3}, inv), ({"Hq": 18}, uns), ({"dt": 2}, uns), ({"scale": -1.0}, inv), ({"scale": float("nan")}, inv),
                     ({"scale": float("inf")}, inv), ({"q": None}, inv), ({"out": None}, inv), ({"ws": None}, inv), ({"q": F + 4}, inv), ({"out": F + 8}, inv),
                     ({"ws": F + 8}, inv), ({"lse": F + 2}, inv), ({"st_t": 510}, uns), ({"st_h": 100}, uns), ({"st_t": 0}, uns),
                     ({"wb": ck._lib.catekv_chunk_attn_workspace_bytes(4, 2, 3) - 1}, ck.ERR_WORKSPACE)):
        assert attend(ck, f, c, **kw) == code, kw
    assert attend(ck, Fake(ck, [2, 300]), c) == inv                          # a list shorter than the chunk
    f.len[0] = 400
    assert attend(ck, f, c) == inv                                           # longer than its capacity
    f.len[0], f.cap[0] = 300, 320
    assert attend(ck, f, c) == inv                                           # a capacity that is no multiple of 128
    assert attend(ck, Fake(ck, [300, 300], caps=False), c) == inv
    g = Fake(ck, [300, 300])
    g.st.d = 64
    assert attend(ck, g, c) == uns


def test_workspace_sizes(ck):
    size = ck._lib.catekv_chunk_attn_workspace_bytes
    assert size(0, 1, 1) == size(4, 3, 1) == size(18, 2, 1) == size(4, 0, 1) == size(4, 2, -1) == 0
    assert 0 < size(4, 2, 0) <= size(4, 2, 1) < size(4, 2, 3) < size(4, 2, 64) < size(4, 2, 65) == size(4, 2, 100000)


def test_chunk_objects(ck):
    c = ck.Chunk([3, 0, 2])
    assert c.n_tokens == 5 and c.start is None and c.struct.B == 3
    c = ck.Chunk([3, 0, 2], [4, 0, 8])
    assert c.n_tokens == 10 and c.start.tolist() == [4, 0, 8]
    assert ck.Chunk([1, 1], [0, 5], 40).n_tokens == 40
    for args in (([-1],), ([2 ** 31],), ([1], [-1]), ([1, 2], [0]), ([1], None, -1), ([1], None, 2 ** 31)):
        with pytest.raises(ck.CatekvError) as e:
            ck.Chunk(*args)
        assert e.value.code == ck.ERR_INVALID_ARG


def fork(ck, f, parent):
    return ck._lib.catekv_fork(C.byref(f.st), np.array(parent, dtype=np.int32).ctypes.data, None)


def truncate(ck, f, drop):
    return ck._lib.catekv_truncate(C.byref(f.st), np.array(drop, dtype=np.int32).ctypes.data, None)


def test_forks_that_are_refused(ck):
    f = Fake(ck, [200, 200, 50, 0], B=4, pages=(3, 3))
    before = f.state()
    assert fork(ck, f, [0, 1, 4, 3]) == fork(ck, f, [0, -1, 2, 3]) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_fork(C.byref(f.st), None, None) == ck.ERR_INVALID_ARG
    assert fork(ck, Fake(ck, [200, 200], B=2), [0, 0]) == ck.ERR_INVALID_ARG  # no pages
    assert fork(ck, f, [0, 0, 0, 3]) == ck.ERR_CAPACITY                       # two pages each for 72 rows, three are there
    assert fork(ck, f, [0, 1, 2, 3]) == ck.OK                                 # nobody continues from another
    f.pages.max_pages = 1
    assert fork(ck, f, [0, 0, 2, 3]) == ck.ERR_CAPACITY                       # a table row of one page
    f.pages.max_pages = 3
    f.st.reserved = 1
    assert fork(ck, f, [0, 0, 2, 3]) == truncate(ck, f, [1, 0, 0, 0]) == ck.ERR_INVALID_ARG
    f.st.reserved = 0
    f.give(0, 7)                                                              # a page that is not there
    assert fork(ck, f, [0, 0, 2, 3]) == ck.ERR_INVALID_ARG
    f.table[0, 0], f.seg_pages[0], f.pages.next_free = -1, 0, 0
    f.seg_pages[1] = 4
    assert fork(ck, f, [0, 0, 2, 3]) == ck.ERR_INVALID_ARG
    f.seg_pages[1] = 0
    assert f.state() == before


def test_truncations_that_are_refused(ck):
    f = Fake(ck, [200, 90], B=2, pages=(8, 4))
    before = f.state()
    assert truncate(ck, f, [-1, 0]) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_truncate(C.byref(f.st), None, None) == ck.ERR_INVALID_ARG
    assert truncate(ck, f, [0, 0]) == ck.OK                                   # nothing to take back
    f.len[1] = -1
    assert truncate(ck, f, [1, 0]) == ck.ERR_INVALID_ARG
    f.len[1] = 90
    # two lists that read the same rows, and no page for the one that would have to leave them
    f.off[1], f.cap[1], f.len[1] = f.off[0], 128, 128
    f.pages.n_pages = 0
    f.len[0] = 200
    assert truncate(ck, f, [100, 0]) == ck.ERR_CAPACITY
    f.off[1], f.cap[1], f.len[1], f.pages.n_pages = 256, 128, 90, 8
    assert f.state() == before


def test_compacting_is_refused(ck):
    call = lambda f: ck._lib.catekv_pages_compact(C.byref(f.st), None, None)
    assert call(Fake(ck, [10])) == ck.ERR_INVALID_ARG
    f = Fake(ck, [128], pages=(8, 4))
    f.give(0, 2, 9)
    assert call(f) == ck.ERR_INVALID_ARG                                      # a page that is not there
    f = Fake(ck, [128], pages=(8, 4))
    f.give(0, 0, 1)
    before = f.table.copy()
    n = C.c_int32(-1)
    assert ck._lib.catekv_pages_compact(C.byref(f.st), C.byref(n), None) == ck.OK and n.value == 2  # they are at the front: nothing moves
    assert np.array_equal(f.table, before) and f.pages.next_free == 2 and f.pages.released == 0


def test_what_fails_on_the_way_changes_nothing(ck):
    """Without a device the first call that needs one fails: the host's tables stay as they were."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    f = Fake(ck, [200, 200, 50, 0], B=4, pages=(9, 3))
    before = f.state()
    assert fork(ck, f, [0, 0, 2, 3]) == truncate(ck, f, [5, 0, 0, 0]) == ck._lib.catekv_pages_reserve(C.byref(f.st), 100, None) == ck.ERR_CUDA
    assert append(ck, f, chunk(ck, [1, 1, 1, 1])) == ck.ERR_CAPACITY          # the last list has no room, and no pages
    assert append(ck, f, chunk(ck, [1, 1, 1, 0])) == attend(ck, f, chunk(ck, [1, 0, 0, 0])) == ck.ERR_CUDA
    assert f.state() == before


def test_binding_refuses(ck):
    class Cache:
        B = 2
    for x in ([1], [1, 2, 3], [-1, 0], [0, 2 ** 31]):
        with pytest.raises(ck.CatekvError) as e:
            ck._per_sequence("x", Cache, x)
        assert e.value.code == ck.ERR_INVALID_ARG


def test_chunks_beyond_the_schedules_count_are_refused(ck):
    """The schedule counts blocks times tiles in 32 bits, and a replayed call may find lists as long as their capacities."""
    n = 1 << 20
    big = Fake(ck, [n] * 64)
    assert attend(ck, big, chunk(ck, [n]), Hq=64, st_t=64 * 128) == ck.ERR_UNSUPPORTED
    roomy = Fake(ck, [2048] * 64, max_new=4 * n)  # 16 blocks of a list, 32 K tiles each once it is full
    assert attend(ck, roomy, chunk(ck, [2048]), Hq=64, st_t=64 * 128, ws=None) == ck.ERR_INVALID_ARG  # fits the count: the next check speaks
    roomy = Fake(ck, [8192] * 512, B=8, max_new=2 * n)  # 512 lists x 512 blocks x 16 K tiles once they are full
    assert attend(ck, roomy, chunk(ck, [8192] * 8), Hq=512, st_t=512 * 128) == ck.ERR_UNSUPPORTED
