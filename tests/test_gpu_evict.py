"""Weighted attention and eviction on the GPU against the oracle.

Tolerances.  Attention: those of the library's decode attention (helpers.py); catekv_decode_attn on the same plan differs by the
roundings of its accumulators alone (some hundred sums, each cut off by up to 2^-23: 1e-4 is far above both), its LSE by those of fp32 sums
in another order.  A weight is a sum of G
exponentials of fp32 numbers: a logit (up to 128 * 2^-23 of the sum of its products' magnitudes, 1e-4 at the very worst, 1e-5 as
a rule) minus the LSE of such logits, so 2e-4 relative per step, plus fp32 additions (2^-24 each).  Eviction copies: exact."""
import numpy as np
import pytest
import torch

import helpers as H
from oracle import catekv_oracle as orc
from workloads import synth

pytestmark = pytest.mark.gpu

W_REL = 2e-4


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def _weights(ck, cache, seed, ties=True):
    """Weights of every list, heavy-tailed, with ties and zeros; what lies behind the lists is a sentinel."""
    g = torch.Generator().manual_seed(seed)
    w = torch.full((max(cache.total_rows, 1),), -5.0)
    for s in range(cache.B * cache.Hkv):
        n, o = int(cache.seg_len[s]), int(cache.seg_off[s])
        x = torch.rand(n, generator=g) ** 8
        if ties:
            x = torch.where(torch.rand(n, generator=g) < 0.5, (x * 16).floor() / 16, x)
        w[o:o + n] = x
    return w.cuda()


def _weighted(ck, cache, q, w, decay, ctas=None, dtype=torch.float32, lse=True):
    plan = ck.DecodePlan(cache, ctas or ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(cache, plan)
    ws = ck.decode_weighted_workspace(cache, q.shape[1], plan)
    ws.fill_(0xFF)
    out = torch.full(q.shape, float("nan"), dtype=dtype, device="cuda")
    ls = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
    ck.catekv_decode_attn_weighted(cache, q, plan, out, w, decay, ws, ls)
    want, wl = torch.empty_like(out), torch.empty(q.shape[:2], device="cuda")
    ck.catekv_decode_attn(cache, q, plan, want, wl)
    tol = 1e-4 if dtype == torch.float32 else 2.0 ** -7  # two bf16 neighbours
    assert (out.float() - want.float()).abs().max() <= tol * want.float().abs().max()
    if ls is not None:
        assert torch.equal(torch.isfinite(ls), torch.isfinite(wl)) and (ls - wl)[torch.isfinite(wl)].abs().max() <= 1e-5
    return out, ls


def _want_weights(oc, q, w0, decay, cache):
    qf = q.cpu().double().numpy()
    G = q.shape[1] // oc.Hkv
    want = w0.double().cpu().numpy().copy()
    for s in range(oc.B * oc.Hkv):
        b, h = divmod(s, oc.Hkv)
        K = orc.bf16_to_f64(oc.k_rows[s])
        o = int(cache.seg_off[s])
        want[o:o + len(K)] = decay * want[o:o + len(K)] + orc.group_attention_weights(qf[b, h * G:h * G + G], K, 128 ** -0.5)
    return want


def _close(w, want, where=""):
    got = w.double().cpu().numpy()
    assert np.array_equal(got[want == -5.0], want[want == -5.0]), (where, "behind the lists")
    err = np.abs(got - want)
    assert np.all(err <= W_REL * np.abs(want) + 1e-30), (where, (err / np.maximum(np.abs(want), 1e-30)).max())


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_weights_every_group_size(ck, G):
    lens = [0, 1, 17, 64, 65, 500, 1500, 3001]
    oc = H.random_cache(2, 4, lens, seed=200 + G)
    cache = H.device_cache_from_oracle(ck, oc, 5)
    q = synth.randn_bf16((2, 4 * G, 128), "cuda", 201, "q", G)
    for ctas, decay in ((1, 1.0), (37, 0.5), (None, 0.9)):
        w0 = _weights(ck, cache, G)
        w = w0.clone()
        _weighted(ck, cache, q, w, decay, ctas, torch.bfloat16 if ctas == 37 else torch.float32, lse=ctas != 1)
        _close(w, _want_weights(oc, q, w0, decay, cache), (G, ctas))


def test_decay_zero_does_not_read_the_old_weights(ck):
    oc = H.random_cache(1, 2, [300, 40], seed=210)
    cache = H.device_cache_from_oracle(ck, oc, 0)
    q = synth.randn_bf16((1, 6, 128), "cuda", 211, "q")
    w = torch.full((cache.total_rows,), float("nan"), device="cuda")
    _weighted(ck, cache, q, w, 0.0)
    for s, n in enumerate((300, 40)):
        o = int(cache.seg_off[s])
        assert abs(float(w[o:o + n].double().sum()) - 1) <= 1e-4 and torch.isnan(w[o + n:o + int(cache.seg_cap[s])]).all()


def test_weights_follow_appends_under_one_plan_and_a_captured_step(ck):
    lens, steps = [60, 200, 0, 128], 6
    oc = H.random_cache(1, 4, lens, seed=220)
    cache = H.device_cache_from_oracle(ck, oc, steps + 1)
    plan = ck.DecodePlan(cache, 24)
    ck.catekv_decode_plan(cache, plan)
    ws = ck.decode_weighted_workspace(cache, 8, plan)
    w = torch.zeros(cache.total_rows, device="cuda")
    q = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    kn, vn = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(1, 8, 128, device="cuda")
    want = w.double().cpu().numpy()

    def new_step(t):
        for x, name, shape in ((q, "q", (1, 8, 128)), (kn, "kn", (1, 4, 128)), (vn, "vn", (1, 4, 128))):
            x.copy_(synth.randn_bf16(shape, "cuda", 221, name, t))
        oc.append(synth.bits(kn), synth.bits(vn))
    new_step(0)
    ck.catekv_append(cache, kn, vn)  # an eager step, then the same step captured
    ck.catekv_decode_attn_weighted(cache, q, plan, out, w, 0.75, ws)
    want = _want_weights(oc, q, torch.from_numpy(want), 0.75, cache)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    before = cache.seg_len.copy()
    with torch.cuda.graph(graph, stream=s):
        ck.catekv_append(cache, kn, vn)
        ck.catekv_decode_attn_weighted(cache, q, plan, out, w, 0.75, ws)
    cache.seg_len[:] = before
    for t in range(1, steps):
        new_step(t)
        ck.catekv_cache_advance(cache)
        graph.replay()
        want = _want_weights(oc, q, torch.from_numpy(want), 0.75, cache)
        ref, _ = orc.decode_attention(oc, synth.bits(q))
        assert H.rel_l2(out.cpu().double().numpy(), ref) <= H.REL_L2
    got = w.double().cpu().numpy()
    # fp32 sums of up to six terms
    assert np.all(np.abs(got - want) <= W_REL * want + 1e-30)


# ---------------------------------------------------------------------------------------------- eviction
def _run_evict(ck, oc, cache, w, mask, budget, sink, local, in_place, max_new=0, idx=True):
    """-> (cache, weights, idx) after the call."""
    n = oc.B * oc.Hkv
    lens = ck.catekv_evict_lengths(cache, mask, budget, sink, local)
    ix = torch.full((n, max(int(lens.max()), 1) + 3), -7, dtype=torch.int32, device="cuda") if idx else None
    if in_place:
        ws = ck.catekv_evict(cache, w, mask, budget, sink, local, idx_out=ix)
        dst, dw = cache, w
    else:
        dst = ck.Cache(oc.B, oc.Hkv, lens, max_new, "cuda")
        dst.k_pool.fill_(3.0)
        dst.v_pool.fill_(3.0)
        dw = torch.full((max(dst.total_rows, 1),), 9.0, device="cuda")
        ws = ck.catekv_evict(cache, w, mask, budget, sink, local, dst, dw, ix)
    assert ck.catekv_workspace_status(ws)["flags"] == 0
    return dst, dw, ix, lens


def _check_evicted(oc, w0, off0, cap0, mask, budget, sink, local, dst, dw, ix, lens, in_place, k0=None, v0=None):
    w0 = w0.cpu().numpy()
    dk, dv, dw = synth.bits(dst.k_pool), synth.bits(dst.v_pool), dw.cpu().numpy()
    assert dst.seg_len_dev.cpu().tolist() == dst.seg_len.tolist() == lens.tolist()
    for s in range(oc.B * oc.Hkv):
        n, o = len(oc.k_rows[s]), int(off0[s])
        rows = orc.evict_indices(w0[o:o + n], sink, local, budget) if mask[s] else np.arange(n)
        t, do, cap = len(rows), int(dst.seg_off[s]), int(dst.seg_cap[s])
        assert lens[s] == t
        assert np.array_equal(dk[do:do + t], oc.k_rows[s][rows]), s
        assert np.array_equal(dv[do:do + t], oc.v_rows[s][rows]), s
        assert np.array_equal(dw[do:do + t], w0[o:o + n][rows], equal_nan=True), s
        if in_place and t == n:
            assert np.array_equal(dw[do + t:do + cap], w0[o + n:o + cap]), s  # not touched
        else:
            assert not dw[do + t:do + cap].any(), s
        if in_place:
            assert np.array_equal(dk[do + t:do + cap], k0[do + t:do + cap]), s  # rows behind the kept ones stay
        else:
            assert np.all(dst.k_pool[do + t:do + cap].float().cpu().numpy() == 3.0), s
        if ix is not None:
            g = ix[s].cpu().numpy()
            assert np.array_equal(g[:t], rows) and np.all(g[t:] == -7), s


LENS = [0, 1, 2, 63, 64, 65, 100, 128, 129, 1000, 1025, 2048, 5000, 300, 64, 777]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("budget,sink,local", [(64, 4, 16), (0, 0, 0), (0, 3, 5), (1, 0, 0), (63, 0, 63), (100, 70, 0), (1024, 4, 64), (1 << 30, 0, 0),
                                               (500, 1, 1)])
def test_evict_against_the_oracle(ck, in_place, budget, sink, local):
    oc = H.random_cache(2, 8, LENS, seed=300)
    cache = H.device_cache_from_oracle(ck, oc, 40)
    mask = np.array([1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1, 0, 1, 1], dtype=np.uint8)
    w = _weights(ck, cache, 301)
    w0, k0 = w.clone(), synth.bits(cache.k_pool).copy()
    res = _run_evict(ck, oc, cache, w, mask, budget, sink, local, in_place, max_new=70)
    _check_evicted(oc, w0, cache.seg_off, cache.seg_cap, mask, budget, sink, local, *res, in_place, k0)
    if not in_place:  # the source is as it was
        assert torch.equal(w, w0) and np.array_equal(synth.bits(cache.k_pool), k0) and cache.seg_len.tolist() == LENS


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["equal", "zeros", "ascending", "descending", "nan", "two", "subnormal"])
def test_evict_weights_that_are_hard_to_rank(ck, in_place, kind):
    lens = [4000, 333, 20000, 33333]  # the last one is longer than the one-CTA selection takes
    oc = H.random_cache(1, 4, lens, seed=310)
    cache = H.device_cache_from_oracle(ck, oc, 0)
    w = torch.zeros(cache.total_rows)
    g = torch.Generator().manual_seed(5)
    for s, n in enumerate(lens):
        o = int(cache.seg_off[s])
        x = torch.arange(n, dtype=torch.float32)
        w[o:o + n] = {"equal": torch.full((n,), 0.125), "zeros": torch.zeros(n), "ascending": x * 1e-3, "descending": (n - x) * 1e-3,
                      "nan": torch.where(torch.rand(n, generator=g) < 0.01, float("nan"),
                                         torch.where(torch.rand(n, generator=g) < 0.01, float("inf"), torch.randn(n, generator=g))),
                      "two": (torch.rand(n, generator=g) < 0.3).float() * 2.0 ** -20,
                      "subnormal": torch.rand(n, generator=g) * 1e-40}[kind]
    w = w.cuda()
    w0, k0 = w.clone(), synth.bits(cache.k_pool).copy()
    mask = np.ones(4, dtype=np.uint8)
    for budget in (150,):
        res = _run_evict(ck, oc, cache, w, mask, budget, 3, 20, in_place)
        _check_evicted(oc, w0, cache.seg_off, cache.seg_cap, mask, budget, 3, 20, *res, in_place, k0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,budget", [(40000, 20000), (70000, 69000), (32768 + 24, 32768), (12400, 5000)])
def test_evict_long_lists(ck, in_place, n, budget):
    lens = [n, 500, n - 1, n // 2]
    oc = H.random_cache(1, 4, lens, seed=320)
    cache = H.device_cache_from_oracle(ck, oc, 10)
    w = _weights(ck, cache, 321)
    w0, k0 = w.clone(), synth.bits(cache.k_pool).copy()
    mask = np.ones(4, dtype=np.uint8)
    res = _run_evict(ck, oc, cache, w, mask, budget, 4, 64, in_place)
    _check_evicted(oc, w0, cache.seg_off, cache.seg_cap, mask, budget, 4, 64, *res, in_place, k0)


@pytest.mark.parametrize("long", [False, True])
def test_a_captured_eviction_replays_on_lists_that_have_grown(ck, long):
    lens = [300, 300, 80] if not long else [300, 20000, 9000]
    oc = H.random_cache(1, 3, lens, seed=330)
    cache = H.device_cache_from_oracle(ck, oc, 60)
    mask = np.array([1, 0, 1], dtype=np.uint8)
    w = _weights(ck, cache, 331)
    ws = ck.evict_workspace(cache)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    ck.catekv_evict(cache, w, mask, 256, 4, 32, ws=ws)  # outside the capture first (launch attributes are set once)
    first = [len(orc.evict_indices(np.zeros(n), 4, 32, 256)) if m else n for n, m in zip(lens, mask)]
    assert cache.seg_len.tolist() == first
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        ck.catekv_evict(cache, w, mask, 256, 4, 32, ws=ws)
    for t in range(20):
        x = synth.randn_bf16((1, 3, 128), "cuda", 332, t)
        ck.catekv_append(cache, x, x)
    grown = cache.seg_len.copy()
    for i in range(3):
        w[int(cache.seg_off[i]):int(cache.seg_off[i]) + int(grown[i])] = torch.rand(int(grown[i]), device="cuda")
    w0, k0, v0 = w.clone(), synth.bits(cache.k_pool).copy(), synth.bits(cache.v_pool).copy()
    graph.replay()
    ck.catekv_cache_sync_lengths(cache)
    k1, w1 = synth.bits(cache.k_pool), w.cpu().numpy()
    for i in range(3):
        o, n = int(cache.seg_off[i]), int(grown[i])
        rows = orc.evict_indices(w0.cpu().numpy()[o:o + n], 4, 32, 256) if mask[i] else np.arange(n)
        assert int(cache.seg_len[i]) == len(rows)
        assert np.array_equal(k1[o:o + len(rows)], k0[o:o + n][rows]) and np.array_equal(w1[o:o + len(rows)], w0.cpu().numpy()[o:o + n][rows])
        assert np.array_equal(synth.bits(cache.v_pool)[o:o + len(rows)], v0[o:o + n][rows])


def test_a_replay_that_outgrows_the_destination_is_cut_and_reported(ck):
    oc = H.random_cache(1, 2, [100, 100], seed=340)
    cache = H.device_cache_from_oracle(ck, oc, 100)
    dst = ck.Cache(1, 2, [100, 100], 0)
    w, dw = _weights(ck, cache, 341), torch.zeros(dst.total_rows, device="cuda")
    mask = np.zeros(2, dtype=np.uint8)
    ws = ck.catekv_evict(cache, w, mask, 50, 0, 0, dst, dw)
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        ck.catekv_evict(cache, w, mask, 50, 0, 0, dst, dw, ws=ws)
    for t in range(40):
        x = synth.randn_bf16((1, 2, 128), "cuda", 342, t)
        ck.catekv_append(cache, x, x)
    graph.replay()
    st = ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)
    assert st["flags"] == ck.STATUS_CAPACITY and st["kernel"] == 6
    assert dst.seg_len_dev.cpu().tolist() == [128, 128]
    for i in range(2):
        assert torch.equal(dst.k_pool[int(dst.seg_off[i]):int(dst.seg_off[i]) + 128], cache.k_pool[int(cache.seg_off[i]):int(cache.seg_off[i]) + 128])


@pytest.mark.parametrize("dtype", [orc.Q8_E4M3, orc.Q8_INT8])
def test_decode_with_weights_then_evict_then_eight_bits(ck, dtype):
    """The calls as they are used together: a few decode steps that accumulate weights, the consistent heads cut back to their budget in
    place, more steps, the cache to 8 bits, and steps on that."""
    B, Hkv, G, sink, local, budget = 2, 4, 4, 4, 32, 200
    lens = [260, 1000, 190, 700, 260, 260, 900, 150]
    mask = np.array([1, 0, 1, 0, 1, 1, 0, 1], dtype=np.uint8)
    oc = H.random_cache(B, Hkv, lens, seed=400)
    cache = H.device_cache_from_oracle(ck, oc, 80)
    plan = ck.DecodePlan(cache, 40)
    ck.catekv_decode_plan(cache, plan)
    ws = ck.decode_weighted_workspace(cache, Hkv * G, plan)
    w = torch.zeros(cache.total_rows, device="cuda")
    out, lse = torch.empty(B, Hkv * G, 128, device="cuda"), torch.empty(B, Hkv * G, device="cuda")

    def token(t):
        q, kn, vn = (synth.randn_bf16((B, h, 128), "cuda", 401, name, t) for name, h in (("q", Hkv * G), ("k", Hkv), ("v", Hkv)))
        oc.append(synth.bits(kn), synth.bits(vn))
        return q, kn, vn
    t = 0
    for part in range(2):
        for _ in range(12):
            q, kn, vn = token(t)
            t += 1
            ck.catekv_append(cache, kn, vn)
            ck.catekv_decode_attn_weighted(cache, q, plan, out, w, 0.9, ws, lse)
            ref, ref_lse = orc.decode_attention(oc, synth.bits(q))
            H.check_attention(out, None, lse, ref, ref_lse, t)
        wv = w.cpu().numpy()
        ck.catekv_evict(cache, w, mask, budget, sink, local)
        for s in range(B * Hkv):
            if mask[s]:
                n, o = len(oc.k_rows[s]), int(cache.seg_off[s])
                rows = orc.evict_indices(wv[o:o + n], sink, local, budget)
                oc.k_rows[s], oc.v_rows[s] = oc.k_rows[s][rows], oc.v_rows[s][rows]
        assert cache.seg_len.tolist() == oc.lengths().tolist()
        if part == 0:  # the plan is for longer lists (the second time it is for lists of the budget's length: still good)
            with pytest.raises(ck.CatekvError) as e:
                ck.catekv_decode_attn_weighted(cache, q, plan, out, w, 0.9, ws, lse)
            assert e.value.code == ck.ERR_INVALID_ARG
            ck.catekv_decode_plan(cache, plan)
    q8 = ck.Q8Cache(B, Hkv, cache.seg_len, 70, dtype)
    ck.catekv_q8_quantize(cache, q8)
    p8 = ck.DecodePlan(q8, 40)
    ck.catekv_q8_decode_plan(q8, p8)
    for i in range(70):
        q, kn, vn = token(t)
        t += 1
        ck.catekv_q8_append(q8, kn, vn)
        if i % 23 == 0:
            ck.catekv_q8_decode_attn(q8, q, p8, out, lse)
            qf = q.cpu().double().numpy()
            for s in range(B * Hkv):
                K, V = orc.q8_rows(oc.k_rows[s], dtype), orc.q8_rows(oc.v_rows[s], dtype)
                b, h = divmod(s, Hkv)
                for g in range(G):
                    o, l = orc.attention(qf[b, h * G + g], K, V, 128 ** -0.5)
                    assert H.rel_l2(out[b, h * G + g].cpu().double().numpy(), o) <= 1e-4 and abs(float(lse[b, h * G + g]) - l) <= 1e-4


def test_two_evictions_on_two_streams(ck):
    """Separate caches and workspaces, lists long enough for clusters of CTAs; in place and into another cache."""
    lens = [30000, 9000, 400]
    mask = np.ones(3, dtype=np.uint8)
    ocs = [H.random_cache(1, 3, lens, seed=500 + i) for i in range(2)]
    caches = [H.device_cache_from_oracle(ck, oc, 5) for oc in ocs]
    ws = [_weights(ck, c, 510 + i) for i, c in enumerate(caches)]
    w0 = [w.clone() for w in ws]
    k0 = [synth.bits(c.k_pool).copy() for c in caches]
    kept = ck.catekv_evict_lengths(caches[1], mask, 3000, 4, 64)
    dst = ck.Cache(1, 3, kept, 0, "cuda")
    dst.k_pool.fill_(3.0)
    dst.v_pool.fill_(3.0)
    dw = torch.full((dst.total_rows,), 9.0, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        ck.catekv_evict(caches[0], ws[0], mask, 3000, 4, 64)
    with torch.cuda.stream(streams[1]):
        ck.catekv_evict(caches[1], ws[1], mask, 3000, 4, 64, dst, dw)
    torch.cuda.synchronize()
    _check_evicted(ocs[0], w0[0], caches[0].seg_off, caches[0].seg_cap, mask, 3000, 4, 64, caches[0], ws[0], None, kept, True, k0[0])
    _check_evicted(ocs[1], w0[1], caches[1].seg_off, caches[1].seg_cap, mask, 3000, 4, 64, dst, dw, None, kept, False)
