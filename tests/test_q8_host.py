"""CPU tests of the 8-bit cache: the oracle's rounding against torch's own types, the plan, the refusals (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import catekv_oracle as orc
from workloads import synth


@pytest.fixture(scope="module")
def ck():
    from paper_2608_30295_b200 import build
    build.build()
    from paper_2608_30295_b200 import binding
    return binding


def test_grids_are_the_types_numbers():
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.q8_grid(orc.Q8_E4M3), e4m3)
    assert np.array_equal(orc.q8_grid(orc.Q8_INT8), np.arange(128))


@pytest.mark.parametrize("dtype", [orc.Q8_E4M3, orc.Q8_INT8])
def test_oracle_rounding_against_torch(dtype):
    # torch rounds a float64 / float32 number to nearest even; the quotient x M / a in float64 is 2^-53 off, borders are 2^-17 away or exact
    x = synth.randn_bf16((64, 128), "cpu", 11, "x")
    num, s = orc.q8_encode(synth.bits(x), dtype)
    M = 448.0 if dtype == orc.Q8_E4M3 else 127.0
    r = x.double() * M / x.double().abs().max()
    want = r.float().to(torch.float8_e4m3fn).double() if dtype == orc.Q8_E4M3 else torch.round(r)
    assert np.array_equal(num, want.numpy())
    assert s == np.float32(float(x.double().abs().max()) / M)


def test_oracle_rounding_hand_worked():
    # a = 127: x M / a = x for int8, so halves go to the even neighbour; a = 448 likewise for e4m3 (17 lies between 16 and 18)
    x = torch.zeros(64, 128)
    x[0, :7] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 3.0])
    num, s = orc.q8_encode(synth.bits(x.bfloat16()), orc.Q8_INT8)
    assert list(num[0, :7]) == [127, 0, 2, 2, 0, -2, 3] and s == 1.0
    x[0, :7] = torch.tensor([448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -17.0, 1.0])
    num, s = orc.q8_encode(synth.bits(x.bfloat16()), orc.Q8_E4M3)
    assert list(num[0, :7]) == [448, 16, 20, 0, 2.0 ** -8, -16, 1] and s == 1.0


def test_oracle_rows_keep_the_unfinished_block():
    x = synth.randn_bf16((70, 128), "cpu", 5, "x")
    got = orc.q8_rows(synth.bits(x), orc.Q8_INT8)
    assert np.array_equal(got[64:], x[64:].double().numpy())
    step = float(x[:64].abs().max()) / 127
    assert 0 < np.abs(got[:64] - x[:64].double().numpy()).max() <= step / 2 * (1 + 1e-6)


def _q8(ck, B, Hkv, lens, max_new=0, dtype=0, d=128):
    off, cap, total = ck.catekv_cache_layout(B, Hkv, lens, max_new)
    seg_len = np.array(lens, dtype=np.int32)
    f = 0x10000  # stands for device memory; nothing dereferences it here
    st = ck.Q8CacheStruct(B, Hkv, d, dtype, total, f, f, f, f, f, f, f, f, off.ctypes.data, cap.ctypes.data, seg_len.ctypes.data, 0, 0)
    return st, (off, cap, seg_len)


def _plan(ck, st, B, Hkv, ctas):
    n = ck._lib.catekv_decode_plan_bytes(B, Hkv, ctas)
    buf = np.zeros(n, dtype=np.uint8)
    rc = ck._lib.catekv_q8_decode_plan(C.byref(st), ctas, buf.ctypes.data, None, n, None)
    return rc, buf


def _tables(buf):
    h = buf[:48].view(np.int32)
    ctas, n_segs, n_items, n_slots = (int(x) for x in h[1:5])
    off_cta, off_items, off_seg = (int(x) for x in h[8:11])
    cta = buf[off_cta:off_cta + 48 * ctas].view(np.int32).reshape(ctas, 12)
    items = buf[off_items:off_items + 32 * n_items].view(np.int32).reshape(n_items, 8)
    segs = buf[off_seg:off_seg + 16 * n_segs].view(np.int32).reshape(n_segs, 4)
    return cta, items, segs, n_slots


@pytest.mark.parametrize("ctas", [1, 3, 37, 296, 1000])
@pytest.mark.parametrize("lens", [[0, 0, 0, 0], [1, 63, 64, 65], [0, 5000, 128, 1], [70001, 64, 63, 4096], [64, 64, 64, 64]])
def test_plan_covers_every_row_once_and_cuts_at_blocks(ck, lens, ctas):
    st, keep = _q8(ck, 2, 2, lens, max_new=5)
    rc, buf = _plan(ck, st, 2, 2, ctas)
    assert rc == ck.OK
    cta, items, segs, n_slots = _tables(buf)
    seen = []
    for lo, hi in cta[:, :2]:
        seen += list(range(lo, hi))
    assert seen == list(range(len(items)))  # consecutive, each item in one CTA
    for s, n in enumerate(lens):
        mine = items[items[:, 0] == s]
        assert mine[0, 1] == 0 and mine[-1, 2] == n and np.array_equal(mine[1:, 1], mine[:-1, 2])
        assert np.all(mine[:, 1] % 64 == 0)
        assert list(mine[:, 6]) == [0] * (len(mine) - 1) + [1]
        assert np.array_equal(mine[:, 4:6].copy().view(np.int64)[:, 0], keep[0][s] + mine[:, 1])
        if len(mine) == 1:
            assert mine[0, 3] == -1 and segs[s, 1] == 1
        else:
            assert list(mine[:, 3]) == list(range(segs[s, 0], segs[s, 0] + len(mine))) and segs[s, 1] == len(mine)
    assert n_slots == sum(len(items[items[:, 0] == s]) for s in range(4) if (items[:, 0] == s).sum() > 1)


def test_plan_shares_rows_evenly(ck):
    st, keep = _q8(ck, 1, 8, [117964, 2048, 117964, 2048, 117964, 2048, 2048, 117964])
    rc, buf = _plan(ck, st, 1, 8, 296)
    cta, items, _, _ = _tables(buf)
    rows = [int((items[lo:hi, 2] - items[lo:hi, 1]).sum()) for lo, hi in cta[:, :2]]
    assert rc == ck.OK and max(rows) <= sum(rows) / 296 * 1.05 + 256


def test_refusals_of_the_plan(ck):
    st, keep = _q8(ck, 1, 2, [100, 200])
    n = ck._lib.catekv_decode_plan_bytes(1, 2, 8)
    buf = np.zeros(n, dtype=np.uint8)
    call = lambda s, ctas=8, size=n, p=buf.ctypes.data: ck._lib.catekv_q8_decode_plan(s, ctas, p, None, size, None)  # noqa: E731
    assert call(C.byref(st)) == ck.OK
    assert call(None) == ck.ERR_INVALID_ARG
    assert call(C.byref(st), ctas=0) == ck.ERR_INVALID_ARG
    assert call(C.byref(st), p=None) == ck.ERR_INVALID_ARG
    assert call(C.byref(st), size=n - 1) == ck.ERR_WORKSPACE
    keep[2][0] = 1000  # longer than its capacity
    assert call(C.byref(st)) == ck.ERR_INVALID_ARG
    keep[2][0] = -1
    assert call(C.byref(st)) == ck.ERR_INVALID_ARG


@pytest.mark.parametrize("field,value,code", [
    ("B", 0, -1), ("Hkv", -1, -1), ("d", 64, -2), ("dtype", 2, -2), ("total_rows", -1, -1), ("total_rows", 128, -1), ("k_pool", None, -1), ("v_pool", None, -1),
    ("k_scale", None, -1), ("v_scale", None, -1), ("k_tail", None, -1), ("v_tail", None, -1), ("seg_off_dev", None, -1),
    ("seg_len_dev", None, -1), ("seg_off", None, -1), ("seg_cap", None, -1), ("seg_len", None, -1), ("k_pool", 0x10008, -1),
    ("v_tail", 0x10004, -1)])
def test_every_call_checks_the_cache(ck, field, value, code):
    f = 0x10000
    st, keep = _q8(ck, 1, 2, [100, 200], max_new=4)
    rc, plan = _plan(ck, st, 1, 2, 8)
    src, keep2 = _bf16(ck, [100, 200])
    setattr(st, field, value)
    assert ck._lib.catekv_q8_append(C.byref(st), f, f, None) == code
    assert ck._lib.catekv_q8_cache_advance(C.byref(st), 1) == code
    assert ck._lib.catekv_q8_quantize(C.byref(src), C.byref(st), None) == code
    assert _plan(ck, st, 1, 2, 8)[0] == code
    assert ck._lib.catekv_q8_decode_attn(C.byref(st), f, 4, 0.0, f, 0, None, plan.ctypes.data, f, plan.size, f, 1 << 30, None) == code


def _bf16(ck, lens, B=1, Hkv=2, max_new=0):
    off, cap, total = ck.catekv_cache_layout(B, Hkv, lens, max_new)
    seg_len = np.array(lens, dtype=np.int32)
    f = 0x10000
    return ck.CacheStruct(B, Hkv, 128, 0, total, f, f, f, f, off.ctypes.data, cap.ctypes.data, seg_len.ctypes.data), (off, cap, seg_len)


def test_segments_must_be_block_aligned(ck):
    st, keep = _q8(ck, 1, 2, [100, 200])
    keep[0][1] = 160
    assert ck._lib.catekv_q8_append(C.byref(st), 0x10000, 0x10000, None) == ck.ERR_INVALID_ARG


def test_refusals_of_append_and_advance(ck):
    st, keep = _q8(ck, 1, 2, [128, 3])
    f = 0x10000
    assert ck._lib.catekv_q8_append(C.byref(st), f, f, None) == ck.ERR_CAPACITY
    assert ck._lib.catekv_q8_append(C.byref(st), None, f, None) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_q8_append(C.byref(st), f, None, None) == ck.ERR_INVALID_ARG
    keep[2][0] = 100
    assert ck._lib.catekv_q8_append(C.byref(st), f + 2, f, None) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_q8_append(C.byref(st), f, f + 8, None) == ck.ERR_INVALID_ARG
    keep[2][0] = 128
    assert list(keep[2]) == [128, 3]
    assert ck._lib.catekv_q8_cache_advance(C.byref(st), 1) == ck.ERR_CAPACITY
    assert ck._lib.catekv_q8_cache_advance(C.byref(st), -1) == ck.ERR_INVALID_ARG
    keep[2][0] = 100
    assert ck._lib.catekv_q8_cache_advance(C.byref(st), 28) == ck.OK and list(keep[2]) == [128, 31]


def test_refusals_of_quantize(ck):
    st, keep = _q8(ck, 1, 2, [128, 3])
    src, keep2 = _bf16(ck, [128, 3])
    q = lambda s: ck._lib.catekv_q8_quantize(s, C.byref(st), None)  # noqa: E731
    assert q(None) == ck.ERR_INVALID_ARG
    big, keep3 = _bf16(ck, [129, 3])
    assert q(C.byref(big)) == ck.ERR_CAPACITY
    other, keep4 = _bf16(ck, [1, 2, 3], Hkv=3)
    assert q(C.byref(other)) == ck.ERR_INVALID_ARG
    src.reserved = 1  # lengths that are upper bounds
    assert q(C.byref(src)) == ck.ERR_INVALID_ARG
    src.reserved = 0
    keep2[2][0] = 300  # longer than its own capacity
    assert q(C.byref(src)) == ck.ERR_INVALID_ARG
    pg = ck.PagesStruct(1, 1, 0, 0, 0x10000, 0x10000, 0x10000, 0x10000, 0x10000, 0x10000)
    keep2[2][0] = 128
    src.pages = C.pointer(pg)
    assert q(C.byref(src)) == ck.ERR_UNSUPPORTED


def test_refusals_of_attention(ck):
    f = 0x10000
    st, keep = _q8(ck, 1, 2, [100, 200])
    rc, plan = _plan(ck, st, 1, 2, 8)
    ws = ck._lib.catekv_decode_workspace_bytes(1, 2, 8)

    def call(q=f, Hq=4, scale=0.0, out=f, od=0, ph=plan.ctypes.data, pd=f, pb=plan.size, w=f, wb=ws):
        return ck._lib.catekv_q8_decode_attn(C.byref(st), q, Hq, scale, out, od, None, ph, pd, pb, w, wb, None)
    for kw in ({"q": None}, {"out": None}, {"ph": None}, {"pd": None}, {"w": None}, {"Hq": 0}, {"Hq": 3}, {"scale": -1.0},
               {"scale": float("inf")}, {"scale": float("nan")}, {"pb": 10}, {"q": f + 2}, {"out": f + 4}, {"w": f + 8}):
        assert call(**kw) == ck.ERR_INVALID_ARG, kw
    assert call(Hq=18) == ck.ERR_UNSUPPORTED and call(od=2) == ck.ERR_UNSUPPORTED
    assert call(pb=plan.size - 1) == ck.ERR_WORKSPACE and call(wb=ws - 1) == ck.ERR_WORKSPACE
    keep[2][0] = 99  # shorter than the plan knows it
    assert call() == ck.ERR_INVALID_ARG
    keep[2][0] = 100
    # the plans of the two kinds of cache are told apart
    src, keep2 = _bf16(ck, [100, 200])
    other = np.zeros_like(plan)
    assert ck._lib.catekv_decode_plan(C.byref(src), 8, other.ctypes.data, None, other.size, None) == ck.OK
    assert call(ph=other.ctypes.data) == ck.ERR_INVALID_ARG
    assert ck._lib.catekv_decode_attn(C.byref(src), f, 4, 0.0, f, 0, None, plan.ctypes.data, f, plan.size, f, ws, None) == ck.ERR_INVALID_ARG


def test_unknown_type_is_refused_by_the_holder(ck):
    with pytest.raises(ck.CatekvError) as e:
        ck.Q8Cache(1, 1, [5], 0, 7, "cpu")
    assert e.value.code == ck.ERR_UNSUPPORTED
