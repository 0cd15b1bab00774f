"""CPU tests of eviction and weighted attention: the oracle by hand, the length rule, the refusals (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import catekv_oracle as orc

F = 0x10000  # stands for device memory; nothing dereferences it here


@pytest.fixture(scope="module")
def ck():
    from paper_2608_30295_b200 import build
    build.build()
    from paper_2608_30295_b200 import binding
    return binding


def test_oracle_by_hand():
    w = np.array([9, 1, 5, 5, 0, 5, 7, 2, 2, 8.0])
    assert list(orc.evict_indices(w, 1, 2, 10)) == list(range(10))
    assert list(orc.evict_indices(w, 1, 2, 6)) == [0, 2, 3, 6, 8, 9]  # 7, then the two first of three that tie
    assert list(orc.evict_indices(w, 1, 2, 3)) == [0, 8, 9] == list(orc.evict_indices(w, 1, 2, 0))
    assert list(orc.evict_indices(w, 4, 6, 3)) == list(range(10))
    assert list(orc.evict_indices(w, 0, 0, 0)) == []
    assert list(orc.evict_indices(np.array([1.0, np.nan, np.inf, -3.0, 0.0]), 0, 0, 3)) == [0, 1, 2]
    assert list(orc.evict_indices(np.array([-1.0, 0.0, -2.0]), 0, 0, 2)) == [0, 1]


def test_oracle_weights_sum_to_one_and_match_torch():
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn(3, 128, generator=g, dtype=torch.float64), torch.randn(50, 128, generator=g, dtype=torch.float64)
    w = orc.group_attention_weights(q.numpy(), k.numpy(), 0.1)
    assert np.allclose(w, torch.softmax(0.1 * q @ k.T, 1).mean(0).numpy(), rtol=1e-12) and abs(w.sum() - 1) < 1e-12
    assert orc.group_attention_weights(q.numpy(), k.numpy()[:0], 0.1).shape == (0,)


def _cache(ck, lens, B=1, Hkv=None, max_new=0):
    Hkv = Hkv or len(lens) // B
    off, cap, total = ck.catekv_cache_layout(B, Hkv, lens, max_new)
    seg_len = np.array(lens, dtype=np.int32)
    st = ck.CacheStruct(B, Hkv, 128, 0, total, F, F, F, F, off.ctypes.data, cap.ctypes.data, seg_len.ctypes.data, None, F)
    return st, (off, cap, seg_len)


@pytest.mark.parametrize("budget,sink,local", [(0, 0, 0), (5, 0, 0), (64, 4, 32), (64, 40, 40), (1000, 4, 64), (2 ** 31 - 1, 0, 0),
                                               (10, 2 ** 30, 2 ** 30 - 1)])
def test_lengths_are_the_oracles(ck, budget, sink, local):
    lens = [0, 1, 63, 64, 65, 80, 81, 500]
    st, keep = _cache(ck, lens)
    mask = np.array([1, 1, 1, 1, 1, 1, 1, 0], dtype=np.uint8)
    out = np.zeros(8, dtype=np.int32)
    assert ck._lib.catekv_evict_lengths(C.byref(st), mask.ctypes.data, budget, sink, local, out.ctypes.data) == ck.OK
    assert list(out) == [len(orc.evict_indices(np.zeros(n), sink, local, budget)) if m else n for n, m in zip(lens, mask)]


def _evict(ck, src, dst, budget=10, sink=2, local=4, w=F, dw=F + 4096, ws=F, wb=1 << 40, mask=None, idx=None, stride=0):
    mask = np.ones(64, dtype=np.uint8) if mask is None else mask
    p = lambda s: None if s is None else C.byref(s)  # noqa: E731
    return ck._lib.catekv_evict(p(src), w, mask.ctypes.data if mask is not False else None, budget, sink, local, p(dst), dw, idx, stride, ws, wb, None)


def _two(ck, lens=(100, 200), dlens=(100, 200)):
    src, k1 = _cache(ck, list(lens))
    dst, k2 = _cache(ck, list(dlens))
    dst.k_pool, dst.v_pool, dst.seg_len_dev = 2 * F, 2 * F, 2 * F
    return src, dst, (k1, k2)


def test_refusals_of_evict(ck):
    src, dst, keep = _two(ck)
    for kw in ({"budget": -1}, {"sink": -1}, {"local": -1}, {"sink": 2 ** 31 - 1, "local": 1}, {"w": None}, {"dw": None}, {"ws": None},
               {"mask": False}, {"w": F, "dw": F}, {"idx": F, "stride": 9}, {"w": F + 2}, {"dw": F + 1}, {"ws": F + 8}, {"idx": F + 2, "stride": 900}):
        assert _evict(ck, src, dst, **kw) == ck.ERR_INVALID_ARG, kw
    assert _evict(ck, None, dst) == ck.ERR_INVALID_ARG and _evict(ck, src, None) == ck.ERR_INVALID_ARG
    assert _evict(ck, src, src) == ck.ERR_INVALID_ARG  # in place with weights elsewhere
    n = ck._lib.catekv_evict_workspace_bytes(1, 2, 256)
    assert n > 0 and _evict(ck, src, dst, wb=n - 1) == ck.ERR_WORKSPACE
    assert ck._lib.catekv_evict_workspace_bytes(0, 2, 5) == 0 and ck._lib.catekv_evict_workspace_bytes(1, 2, -1) == 0
    src2, dst2, keep2 = _two(ck, dlens=(100, 100))
    assert _evict(ck, src2, dst2, budget=129) == ck.ERR_CAPACITY
    for name in ("k_pool", "v_pool", "seg_len_dev"):  # two caches that share memory
        src3, dst3, keep3 = _two(ck)
        setattr(dst3, name, F)
        assert _evict(ck, src3, dst3) == ck.ERR_INVALID_ARG, name
    for which in (0, 1):
        a = list(_two(ck))
        a[which].seg_cap_dev = None
        assert _evict(ck, a[0], a[1]) == ck.ERR_INVALID_ARG
        pg = ck.PagesStruct(1, 1, 0, 0, F, F, F, F, F, F)
        a = list(_two(ck))
        a[which].pages = C.pointer(pg)
        assert _evict(ck, a[0], a[1]) == ck.ERR_UNSUPPORTED
    src, dst, keep = _two(ck)
    src.reserved = 1  # lengths that are upper bounds
    assert _evict(ck, src, dst) == ck.ERR_INVALID_ARG
    src, dst, keep = _two(ck)
    keep[0][2][0] = 129
    assert _evict(ck, src, dst) == ck.ERR_INVALID_ARG
    other, keep4 = _cache(ck, [1, 2, 3])
    other.k_pool = other.v_pool = other.seg_len_dev = 2 * F
    src, dst, keep = _two(ck)
    assert _evict(ck, src, other) == ck.ERR_INVALID_ARG
    big, keep5 = _cache(ck, [5] * 2052, B=513, Hkv=4)
    big2, keep6 = _cache(ck, [5] * 2052, B=513, Hkv=4)
    big2.k_pool, big2.v_pool, big2.seg_len_dev = 2 * F, 2 * F, 2 * F
    assert _evict(ck, big, big2, mask=np.ones(2052, dtype=np.uint8)) == ck.ERR_UNSUPPORTED


def test_refusals_of_weighted_attention(ck):
    st, keep = _cache(ck, [100, 200])
    n = ck._lib.catekv_decode_plan_bytes(1, 2, 8)
    plan = np.zeros(n, dtype=np.uint8)
    assert ck._lib.catekv_decode_plan(C.byref(st), 8, plan.ctypes.data, None, n, None) == ck.OK
    ws = ck._lib.catekv_decode_weighted_workspace_bytes(1, 4, 2, 8, st.total_rows)
    assert ws > 2 * st.total_rows * 4 + ck._lib.catekv_decode_workspace_bytes(1, 2, 8)
    assert ck._lib.catekv_decode_weighted_workspace_bytes(1, 5, 2, 8, 100) == 0

    def call(q=F, Hq=4, scale=0.0, out=F, od=0, w=F, decay=1.0, ph=plan.ctypes.data, pd=F, pb=n, wsp=F, wb=ws):
        return ck._lib.catekv_decode_attn_weighted(C.byref(st), q, Hq, scale, out, od, None, w, decay, ph, pd, pb, wsp, wb, None)
    for kw in ({"q": F + 2}, {"out": F + 4}, {"wsp": F + 8}, {"w": F + 1}, {"q": None}, {"out": None}, {"w": None}, {"ph": None}, {"pd": None}, {"wsp": None}, {"Hq": 0}, {"Hq": 3}, {"decay": -0.1},
               {"decay": 1.5}, {"decay": float("nan")}, {"scale": -1.0}, {"pb": 10}):
        assert call(**kw) == ck.ERR_INVALID_ARG, kw
    assert call(wb=ws - 1) == ck.ERR_WORKSPACE and call(pb=n - 1) == ck.ERR_WORKSPACE
    keep[2][1] = 199  # shorter than the plan knows it
    assert call() == ck.ERR_INVALID_ARG
    keep[2][1] = 200
    st.reserved = 1  # lengths that are upper bounds
    assert call() == ck.ERR_INVALID_ARG
    st.reserved = 0
    assert call(Hq=18, wb=1 << 40) == ck.ERR_UNSUPPORTED and call(od=7) == ck.ERR_UNSUPPORTED
    pg = ck.PagesStruct(1, 1, 0, 0, F, F, F, F, F, F)
    st.pages = C.pointer(pg)
    assert call() == ck.ERR_UNSUPPORTED


def test_counts_past_int32_are_refused_by_the_binding(ck):
    cache = type("C", (), {"B": 1, "Hkv": 2})()
    for bad in ((2 ** 32, 0, 0), (5, 2 ** 31, 0), (5, 0, -1)):
        with pytest.raises(ck.CatekvError) as e:
            ck.catekv_evict_lengths(cache, [1, 1], *bad)
        assert e.value.code == ck.ERR_INVALID_ARG
