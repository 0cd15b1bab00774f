"""The 8-bit cache on the GPU against the oracle: codes and scales exact, attention over what they stand for.

Tolerances.  Codes are exact (a border between two codes is met exactly or missed by 2^-16 of the quotient, see the oracle), scales are one
IEEE division.  Attention: codes, bf16 rows and queries enter the products exactly; an fp32 sum of 128 products errs by at most
128 * 2^-23 of the sum of their magnitudes, about 1.1 * 7.2 on the scaled logit for N(0, 1) rows, so a probability by 2^-16 * 8 = 1.2e-4 at the
very worst and by the square root of that count (1e-5) as a rule; pairs of 16 and more bits (2^-17) and exp2 (2^-22) stay below it.
So: relative L2 <= 1e-4, |difference| <= 1e-4 * max |V|, LSE 1e-4; a bf16 output is the fp32 output rounded once, bit for bit."""
import numpy as np
import pytest
import torch

import helpers as H
from oracle import catekv_oracle as orc
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


TYPES = [orc.Q8_E4M3, orc.Q8_INT8]


def _src(ck, rows_k, rows_v, B, Hkv, max_new=0, behind=float("nan")):
    """bf16 rows per segment -> Cache; what lies behind a list is NaN."""
    lens = [len(r) for r in rows_k]
    cache = ck.Cache(B, Hkv, lens, max_new)
    cache.k_pool.fill_(behind)
    cache.v_pool.fill_(behind)
    for s, n in enumerate(lens):
        o = int(cache.seg_off[s])
        cache.k_pool[o:o + n], cache.v_pool[o:o + n] = rows_k[s].cuda(), rows_v[s].cuda()
    cache.set_lengths(lens)
    return cache


def _rows(lens, seed, scale=1.0):
    k = [(synth.randn_bf16((n, 128), "cpu", seed, "k", i).float() * scale).bfloat16() for i, n in enumerate(lens)]
    v = [(synth.randn_bf16((n, 128), "cpu", seed, "v", i).float() * scale).bfloat16() for i, n in enumerate(lens)]
    return k, v


def _nan_like(c):
    """Codes, scales and tails that no list covers: NaN (0x7f as e4m3, 127 as int8)."""
    for t in (c.k_pool, c.v_pool):
        t.view(torch.uint8).fill_(0x7F)
    for t in (c.k_scale, c.v_scale, c.k_tail, c.v_tail):
        t.fill_(float("nan"))


def _quantized(ck, k, v, B, Hkv, dtype, max_new=64):
    src = _src(ck, k, v, B, Hkv)
    dst = ck.Q8Cache(B, Hkv, [len(r) for r in k], max_new, dtype)
    _nan_like(dst)
    ck.catekv_q8_quantize(src, dst)
    return dst


def _numbers(pool):
    return (pool if pool.dtype == torch.int8 else pool.float()).double().cpu().numpy()


def _check_codes(c, k, v, dtype):
    """Every code, scale, tail row and length; and that nothing else was written."""
    n_segs = len(k)
    assert c.seg_len_dev.cpu().tolist() == c.seg_len.tolist() == [len(r) for r in k]
    for rows, pool, scale, tail in ((k, c.k_pool, c.k_scale, c.k_tail), (v, c.v_pool, c.v_scale, c.v_tail)):
        num, raw = _numbers(pool), pool.view(torch.uint8).cpu().numpy()
        sc, tl = scale.cpu().numpy(), tail.cpu()
        for s in range(n_segs):
            n, o = len(rows[s]), int(c.seg_off[s])
            full = n // 64 * 64
            for r in range(0, full, 64):
                want, ws = orc.q8_encode(synth.bits(rows[s][r:r + 64]), dtype)
                assert np.array_equal(num[o + r:o + r + 64], want), (s, r)
                assert np.array_equal(sc[(o + r) // 64], ws, equal_nan=True), (s, r)
            assert np.array_equal(synth.bits(tl[s, :n - full]), synth.bits(rows[s][full:])), s
            assert torch.isnan(tl[s, n - full:]).all(), (s, "behind the tail")
            assert np.all(raw[o + full:o + int(c.seg_cap[s])] == 0x7F), (s, "behind the blocks")
            assert np.all(np.isnan(sc[(o + full) // 64:(o + int(c.seg_cap[s])) // 64])), s


LENS = [0, 1, 63, 64, 65, 127, 128, 200]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -120, 2.0 ** 100, 37.0])
def test_quantize_is_exact(ck, dtype, scale):
    k, v = _rows(LENS, 3, scale)
    _check_codes(_quantized(ck, k, v, 2, 4, dtype), k, v, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_borders_between_codes(ck, dtype):
    # every bf16 number of a few binades under largest values that put many of them on the border of two codes (a = M 2^j: x M / a = x 2^-j)
    # or next to one
    M = 448.0 if dtype == orc.Q8_E4M3 else 127.0
    x = (torch.arange(64 * 128, dtype=torch.int32) + 0x3A00).to(torch.int16).view(torch.bfloat16).float()  # 2^-11 .. 2^5 x 1.0 .. 1.99
    k, v = [], []
    for a in (M, M / 4, M * 8, 129.0, 131.0, 251.0, 255.0, 253.0 / 64):
        y = torch.where(x <= a, x, x * 2.0 ** -40).bfloat16().reshape(64, 128).clone()
        y[0, 0] = a
        y[1::2] *= -1
        k.append(y)
        v.append(y.flip(0).contiguous())
    _check_codes(_quantized(ck, k, v, 2, 4, dtype), k, v, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_zeros_largest_and_smallest_numbers(ck, dtype):
    z = torch.zeros(64, 128).bfloat16()
    big = synth.randn_bf16((64, 128), "cpu", 9, "b").clone()
    big[5, 7] = 3.3895313892515355e38
    small = (torch.arange(64 * 128) % 200).to(torch.int16).view(torch.bfloat16).reshape(64, 128)  # subnormals
    one = z.clone()
    one[63, 127] = -1e-30
    k, v = [z, big, small, one], [one, small, big, z]
    _check_codes(_quantized(ck, k, v, 1, 4, dtype), k, v, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_block_that_is_not_finite(ck, dtype, bad):
    k, v = _rows([192, 192, 130], 4)
    k[0][70, 3] = bad      # block 1 of segment 0
    v[1][64 * 3 - 1, 127] = bad
    k[2][129, 0] = bad     # a tail row
    c = _quantized(ck, k, v, 1, 3, dtype)
    ks, vs = c.k_scale.cpu(), c.v_scale.cpu()
    o = c.seg_off
    assert torch.isnan(ks[o[0] // 64 + 1]) and torch.isfinite(ks[[o[0] // 64, o[0] // 64 + 2]]).all() and torch.isfinite(vs[o[0] // 64:o[0] // 64 + 3]).all()
    assert torch.isnan(vs[o[1] // 64 + 2]) and torch.isfinite(ks[o[1] // 64:o[1] // 64 + 3]).all()
    q = synth.randn_bf16((1, 6, 128), "cuda", 8, "q")
    for ctas in (1, 5, 296):
        out, lse = _attend(ck, c, q, ctas)
        assert torch.isnan(out[:, :4]).any(dim=2).all(), ctas
        # the tail is bf16: an infinite key there has the logit +-inf, and exp(-inf) = 0 takes it out of a head's sum
        gone = (q[0, 4:, 0].float() * bad == float("-inf")).cpu()
        assert torch.equal(torch.isnan(out[0, 4:]).any(dim=1).cpu(), ~gone), ctas
    k2, v2 = _rows([192, 192, 130], 4)
    v2[0][0, 0] = bad
    c = _quantized(ck, k2, v2, 1, 3, dtype)
    out, lse = _attend(ck, c, q, 7)
    assert torch.isnan(out[:, :2]).all() and torch.isfinite(out[:, 2:]).all() and torch.isfinite(lse[:, 2:]).all()


def _attend(ck, c, q, ctas=None, sm_scale=0.0, dtype=torch.float32, plan=None):
    if plan is None:
        plan = ck.DecodePlan(c, ctas or ck.catekv_q8_decode_num_ctas())
        plan.ws.fill_(0xFF)
        ck.catekv_q8_decode_plan(c, plan)
    out = torch.full(q.shape, float("nan"), dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    ck.catekv_q8_decode_attn(c, q, plan, out, lse, sm_scale)
    return out, lse


def _oracle(k, v, q, B, Hkv, dtype, sm_scale=0.0):
    G = q.shape[1] // Hkv
    qf = q.cpu().double().numpy()
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    vmax = 0.0
    for b in range(B):
        for h in range(Hkv):
            kk, vv = orc.q8_rows(synth.bits(k[b * Hkv + h]), dtype), orc.q8_rows(synth.bits(v[b * Hkv + h]), dtype)
            vmax = max(vmax, np.abs(vv).max(initial=0.0))
            for g in range(G):
                if len(kk):
                    out[b, h * G + g], lse[b, h * G + g] = orc.attention(qf[b, h * G + g], kk, vv, sm_scale or 128 ** -0.5)
    return out, lse, vmax


def _check_attention(out, lse, ref, where=""):
    r, rl, vmax = ref
    g = out.double().cpu().numpy()
    assert not np.isnan(g).any(), where
    assert H.rel_l2(g, r) <= 1e-4, (where, H.rel_l2(g, r))
    assert H.max_abs(g, r) <= 1e-4 * max(vmax, 1e-30), (where, H.max_abs(g, r))
    gl = lse.double().cpu().numpy()
    fin = np.isfinite(rl)
    assert np.array_equal(np.isfinite(gl), fin) and np.all(gl[~fin] == -np.inf), where
    assert np.all(np.abs(gl[fin] - rl[fin]) <= 1e-4), (where, np.abs(gl[fin] - rl[fin]).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_attention_every_group_size(ck, dtype, G):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 95, 96, 97, 128, 500, 1024, 2000, 3333]
    k, v = _rows(lens, 20 + G)
    c = _quantized(ck, k, v, 2, 8, dtype)
    q = synth.randn_bf16((2, 8 * G, 128), "cuda", 21, "q", G)
    ref = _oracle(k, v, q, 2, 8, dtype)
    for ctas in (1, 13, None):
        out, lse = _attend(ck, c, q, ctas)
        _check_attention(out, lse, ref, (dtype, G, ctas))
        o16, _ = _attend(ck, c, q, ctas, dtype=torch.bfloat16)
        assert np.array_equal(synth.bits(o16.cpu()), synth.bits(out.bfloat16().cpu()))
    again, _ = _attend(ck, c, q)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 64, 66, 129, 4097])
def test_attention_single_segment(ck, dtype, n):
    k, v = _rows([n], 40 + n)
    c = _quantized(ck, k, v, 1, 1, dtype)
    q = synth.randn_bf16((1, 3, 128), "cuda", 41, "q")
    ref = _oracle(k, v, q, 1, 1, dtype, 0.3)
    for ctas in (1, 2, 65, 300):
        out, lse = _attend(ck, c, q, ctas, sm_scale=0.3)
        _check_attention(out, lse, ref, (n, ctas))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("qs,ks,vs", [(2.0 ** 60, 2.0 ** -60, 1.0), (2.0 ** -100, 2.0 ** 100, 2.0 ** 90), (1.0, 1.0, 2.0 ** -110), (30.0, 1.0, 1.0)])
def test_attention_scales_far_from_one(ck, dtype, qs, ks, vs):
    lens = [200, 64, 40, 777]
    k, v = _rows(lens, 50)
    k = [(x.float() * ks).bfloat16() for x in k]
    v = [(x.float() * vs).bfloat16() for x in v]
    c = _quantized(ck, k, v, 1, 4, dtype)
    q = (synth.randn_bf16((1, 8, 128), "cpu", 51, "q").float() * qs).bfloat16().cuda()
    r, rl, vmax = _oracle(k, v, q, 1, 4, dtype)
    out, lse = _attend(ck, c, q, 9)
    if qs == 30.0:  # logits of some hundreds: their error grows with them (128 2^-23 of 30 * 7.2), and so does the LSE's
        assert H.rel_l2(out.cpu().double().numpy(), r) <= 30 * 1e-4 and np.abs(lse.cpu().numpy() - rl).max() <= 30 * 1e-4
    else:
        _check_attention(out, lse, (r, rl, vmax))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_blocks_of_very_different_scales(ck, dtype):
    # a block's V from 2^-40 to 2^40: the accumulators' unit grows, stays and shrinks; K alike in the last segment
    k, v = _rows([64 * 9 + 20, 64 * 9 + 20, 64 * 6], 60)
    for i, e in enumerate((-20, 20, 0, 40, -40, 3, -3, 39, 1)):
        v[0][64 * i:64 * i + 64] *= 2.0 ** e
        v[1][64 * i:64 * i + 64] *= 2.0 ** -e
    for i, e in enumerate((-3, 1, -10, 2, 0, -20)):
        k[2][64 * i:64 * i + 64] *= 2.0 ** e
    v[0][100:120] = 0
    v[1][64:128] = 0  # a block of zeros
    c = _quantized(ck, k, v, 1, 3, dtype)
    q = synth.randn_bf16((1, 12, 128), "cuda", 61, "q")
    r, rl, vmax = _oracle(k, v, q, 1, 3, dtype)
    for ctas in (1, 4, 40):
        out, lse = _attend(ck, c, q, ctas)
        g = out.double().cpu().numpy()
        for h in range(3):
            assert H.rel_l2(g[:, 4 * h:4 * h + 4], r[:, 4 * h:4 * h + 4]) <= 1e-4, (ctas, h)
        assert np.abs(lse.double().cpu().numpy() - rl).max() <= 1e-4 * 4  # logits up to four times as large


@pytest.mark.parametrize("dtype", TYPES)
def test_queries_with_elements_far_apart(ck, dtype):
    # within a head 2^29 and more apart (the smallest fall out of f16, 2^-40 of the largest), zero heads, one element alone
    k, v = _rows([333, 129], 70)
    c = _quantized(ck, k, v, 1, 2, dtype)
    q = synth.randn_bf16((1, 8, 128), "cpu", 71, "q")
    q[0, 0, ::2] *= 2.0 ** -35
    q[0, 1] = 0
    q[0, 2] = 0
    q[0, 2, 17] = 3.0
    q[0, 3] *= torch.exp2(-torch.arange(128) / 3.0)
    q = q.cuda()
    out, lse = _attend(ck, c, q, 3)
    _check_attention(out, lse, _oracle(k, v, q, 1, 2, dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_append_completes_blocks_and_equals_quantize(ck, dtype):
    """70 appends: codes, scales and tails are those of a cache quantised at once; attention along the way."""
    lens, steps = [0, 1, 60, 63, 64, 127, 300], 70
    full_k, full_v = _rows([n + steps for n in lens], 80)
    c = _quantized(ck, [x[:n] for x, n in zip(full_k, lens)], [x[:n] for x, n in zip(full_v, lens)], 1, 7, dtype, max_new=steps)
    plan = ck.DecodePlan(c, 20)
    ck.catekv_q8_decode_plan(c, plan)
    q = synth.randn_bf16((1, 14, 128), "cuda", 81, "q")
    for t in range(steps):
        kn = torch.stack([x[n + t] for x, n in zip(full_k, lens)]).reshape(1, 7, 128).cuda()
        vn = torch.stack([x[n + t] for x, n in zip(full_v, lens)]).reshape(1, 7, 128).cuda()
        ck.catekv_q8_append(c, kn, vn)
        if t in (0, 1, 3, 35, 63, 64, 69):
            k, v = [x[:n + t + 1] for x, n in zip(full_k, lens)], [x[:n + t + 1] for x, n in zip(full_v, lens)]
            out, lse = _attend(ck, c, q, plan=plan)  # the plan of the start follows the lists
            _check_attention(out, lse, _oracle(k, v, q, 1, 7, dtype), t)
    # what is left in a tail behind a completed block is the block's own rows; everything else as if quantised at once
    want = _quantized(ck, full_k, full_v, 1, 7, dtype, max_new=0)
    for s, n in enumerate(lens):
        n += steps
        f, o, w = n // 64 * 64, int(c.seg_off[s]), int(want.seg_off[s])
        for a, b in ((c.k_pool, want.k_pool), (c.v_pool, want.v_pool)):
            assert torch.equal(a.view(torch.uint8)[o:o + f], b.view(torch.uint8)[w:w + f]), s
        for a, b in ((c.k_scale, want.k_scale), (c.v_scale, want.v_scale)):
            assert torch.equal(a[o // 64:(o + f) // 64], b[w // 64:(w + f) // 64]), s
        assert torch.equal(c.k_tail[s, :n - f], want.k_tail[s, :n - f]) and torch.equal(c.v_tail[s, :n - f], want.v_tail[s, :n - f]), s
    assert c.seg_len_dev.cpu().tolist() == c.seg_len.tolist() == [n + steps for n in lens]


@pytest.mark.parametrize("dtype", TYPES)
def test_a_plan_for_longer_lists_is_refused(ck, dtype):
    k, v = _rows([1000, 640, 130], 90)
    c = _quantized(ck, k, v, 1, 3, dtype)
    plan = ck.DecodePlan(c, 12)
    ck.catekv_q8_decode_plan(c, plan)
    q = synth.randn_bf16((1, 6, 128), "cuda", 91, "q")
    k2, v2 = _rows([1000, 0, 130], 92)
    ck.catekv_q8_quantize(_src(ck, k2, v2, 1, 3), c)
    with pytest.raises(ck.CatekvError) as e:
        _attend(ck, c, q, plan=plan)
    assert e.value.code == ck.ERR_INVALID_ARG
    ck.catekv_q8_decode_plan(c, plan)
    out, lse = _attend(ck, c, q, plan=plan)
    _check_attention(out, lse, _oracle(k2, v2, q, 1, 3, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,ctas", [(64 * 60, 15), (64 * 64, 16), (64 * 68, 17), (64 * 31, 31), (64 * 32, 32), (64 * 33, 33), (64 * 80, 80), (5000, 296), (64 * 32 - 1, 200)])
def test_pieces_merged_in_the_kernel_and_by_the_combine_pass(ck, dtype, n, ctas):
    # around the number of pieces up to which the CTA that delivers the last one merges; several calls under one plan
    lens = [n, 100, n // 2, 0]
    k, v = _rows(lens, 140)
    c = _quantized(ck, k, v, 1, 4, dtype)
    plan = ck.DecodePlan(c, ctas)
    plan.ws.fill_(0xFF)
    ck.catekv_q8_decode_plan(c, plan)
    for i in range(4):
        q = synth.randn_bf16((1, 20, 128), "cuda", 141, "q", i)
        out, lse = _attend(ck, c, q, plan=plan)
        _check_attention(out, lse, _oracle(k, v, q, 1, 4, dtype), (n, ctas, i))
        assert all(torch.equal(out, _attend(ck, c, q, plan=plan)[0]) for _ in range(20))  # whoever comes last


@pytest.mark.parametrize("dtype", TYPES)
def test_a_captured_step_replays(ck, dtype):
    lens, steps = [70, 126, 5], 8
    k, v = _rows([n + steps for n in lens], 100)
    c = _quantized(ck, [x[:n] for x, n in zip(k, lens)], [x[:n] for x, n in zip(v, lens)], 1, 3, dtype, max_new=steps)
    plan = ck.DecodePlan(c, 8)
    ck.catekv_q8_decode_plan(c, plan)
    q = synth.randn_bf16((1, 9, 128), "cuda", 101, "q")
    kn, vn = torch.zeros(1, 3, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 3, 128, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty(1, 9, 128, device="cuda"), torch.empty(1, 9, device="cuda")
    _attend(ck, c, q, plan=plan)  # first call outside the capture
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ck.catekv_q8_append(c, kn, vn)
        ck.catekv_q8_decode_attn(c, q, plan, out, lse)
    c.seg_len[:] = lens  # the capture counted its append; nothing has run yet
    for t in range(steps):
        kn.copy_(torch.stack([x[n + t] for x, n in zip(k, lens)]).reshape(1, 3, 128))
        vn.copy_(torch.stack([x[n + t] for x, n in zip(v, lens)]).reshape(1, 3, 128))
        ck.catekv_q8_cache_advance(c)
        graph.replay()
        ref = _oracle([x[:n + t + 1] for x, n in zip(k, lens)], [x[:n + t + 1] for x, n in zip(v, lens)], q, 1, 3, dtype)
        _check_attention(out, lse, ref, t)
    assert c.seg_len_dev.cpu().tolist() == c.seg_len.tolist()


def test_many_short_segments_on_another_stream(ck):
    B, Hkv = 64, 8
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 150, B * Hkv).tolist()
    k, v = _rows(lens, 110)
    c = _quantized(ck, k, v, B, Hkv, orc.Q8_INT8, max_new=0)
    q = synth.randn_bf16((B, Hkv * 2, 128), "cuda", 111, "q")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out, lse = _attend(ck, c, q)
    s.synchronize()
    _check_attention(out, lse, _oracle(k, v, q, B, Hkv, orc.Q8_INT8))


def test_offsets_past_32_bits(ck):
    """The second segment begins behind 2^32 bytes of codes (and 2^33 of the source's rows)."""
    n = 2 ** 25 + 128
    off, cap, total = ck.catekv_cache_layout(1, 2, [n, 300], 0)
    assert int(off[1]) * 128 > 2 ** 32
    src = ck.Cache(1, 2, [n, 300], 0)
    k, v = _rows([70, 300], 120)
    for s in range(2):
        o = int(src.seg_off[s])
        src.k_pool[o:o + len(k[s])], src.v_pool[o:o + len(v[s])] = k[s].cuda(), v[s].cuda()
    src.set_lengths([70, 300])
    c = ck.Q8Cache(1, 2, [n, 300], 0, ck.Q8_E4M3)
    ck.catekv_q8_quantize(src, c)
    q = synth.randn_bf16((1, 8, 128), "cuda", 121, "q")
    out, lse = _attend(ck, c, q)
    _check_attention(out, lse, _oracle(k, v, q, 1, 2, orc.Q8_E4M3))


def test_refusals_leave_everything_as_it_was(ck):
    k, v = _rows([128, 7], 130)
    c = _quantized(ck, k, v, 1, 2, orc.Q8_INT8, max_new=0)
    kn = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_q8_append(c, kn, kn)
    assert e.value.code == ck.ERR_CAPACITY and c.seg_len.tolist() == [128, 7]
    _check_codes(c, k, v, orc.Q8_INT8)
    bf = _src(ck, k, v, 1, 2)
    plan = ck.DecodePlan(bf, 4)
    ck.catekv_decode_plan(bf, plan)
    q = synth.randn_bf16((1, 4, 128), "cuda", 131, "q")
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_q8_decode_attn(c, q, plan, torch.empty(1, 4, 128, device="cuda"))
    assert e.value.code == ck.ERR_INVALID_ARG
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_q8_decode_attn(c, q.cpu(), plan, torch.empty(1, 4, 128, device="cuda"))
    assert e.value.code == ck.ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G", [3, 4, 5])
def test_long_shares(ck, dtype, G):
    # one CTA with a long share: the variant that long streams take, against the same rows shared out over many CTAs and the oracle
    lens = [9000, 5, 4999, 64]
    k, v = _rows(lens, 150)
    c = _quantized(ck, k, v, 1, 4, dtype)
    q = synth.randn_bf16((1, 4 * G, 128), "cuda", 151, "q", G)
    ref = _oracle(k, v, q, 1, 4, dtype)
    for ctas in (1, 2, 3, 100):
        out, lse = _attend(ck, c, q, ctas)
        _check_attention(out, lse, ref, ctas)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G", [4, 6])
def test_infinite_keys_in_a_tail(ck, dtype, G):
    # every tail row of a list holds an infinity: heads for which its logit is -inf see the block alone, the others NaN
    lens = [66, 64 * 5 + 33, 65]
    k, v = _rows(lens, 160)
    for s, n in enumerate(lens):
        k[s][n // 64 * 64:, 0] = float("inf")
    c = _quantized(ck, k, v, 1, 3, dtype)
    q = synth.randn_bf16((1, 3 * G, 128), "cuda", 161, "q", G)
    full = [n // 64 * 64 for n in lens]
    r, rl, vmax = _oracle([x[:n] for x, n in zip(k, full)], [x[:n] for x, n in zip(v, full)], q, 1, 3, dtype)
    gone = (q[0, :, 0] < 0).cpu().numpy()
    assert gone.any() and not gone.all()
    for ctas in (1, 3, 60):
        out, lse = _attend(ck, c, q, ctas)
        g = out[0].double().cpu().numpy()
        assert np.isnan(g[~gone]).any(axis=1).all()
        assert H.rel_l2(g[gone], r[0][gone]) <= 1e-4 and np.abs(lse[0].cpu().numpy()[gone] - rl[0][gone]).max() <= 1e-4


@pytest.mark.parametrize("ctas", [40, 296])
def test_two_streams_with_a_plan_and_a_workspace_each(ck, ctas):
    lens = [2000, 700, 64, 1500]
    k, v = _rows(lens, 170)
    c = _quantized(ck, k, v, 1, 4, orc.Q8_E4M3)
    plans = [ck.DecodePlan(c, ctas) for _ in range(2)]
    for p in plans:
        ck.catekv_q8_decode_plan(c, p)
    qs = [synth.randn_bf16((1, 16, 128), "cuda", 171, "q", i) for i in range(2)]
    want = [_attend(ck, c, q, ctas)[0] for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty(50, 1, 16, 128, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(50):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                ck.catekv_q8_decode_attn(c, qs[s], plans[s], outs[s][i])
    torch.cuda.synchronize()
    for s in range(2):
        assert all(torch.equal(outs[s][i], want[s]) for i in range(50))
