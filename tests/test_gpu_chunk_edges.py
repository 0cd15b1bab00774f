"""Chunk calls where they can go wrong: infinities and NaN, strides and orders, captured and replayed calls, streams, far offsets, waits that run
out, what a list has no room for, and the page calls' larger and rarer forms."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import D, check, get_rows, make_cache, reference
from test_gpu_pages import Model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def queries(T, Hq, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(T, Hq, D, generator=g, device="cuda").bfloat16()


def run(ck, cache, n_new, q, start=None, n_tokens=None, dtype=torch.float32, **kw):
    chunk = ck.Chunk(n_new, start, n_tokens)
    out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=dtype), torch.full(q.shape[:2], 3.0, device="cuda")
    ws = ck.catekv_chunk_attn(cache, chunk, q, out, lse, **kw)
    assert ck.catekv_workspace_status(ws)["flags"] == 0
    return out, lse


def poke(cache, s, row, col, value, what):
    """One element of K or V of list s."""
    cap, off = int(cache.seg_cap[s]), int(cache.seg_off[s])
    pool, ovf = (cache.k_pool, cache.pages.k_ovf) if what == "k" else (cache.v_pool, cache.pages.v_ovf)
    if row < cap:
        pool[off + row, col] = value
    else:
        ovf[int(cache.pages.table[s, (row - cap) // 64]) * 64 + (row - cap) % 64, col] = value


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,base,extra,m", [(4, 128, 60, 40), (1, 0, 300, 290), (8, 500, 0, 9), (3, 256, 200, 150)])
def test_an_infinity_or_a_nan_in_a_new_row_reaches_who_sees_it(ck, G, base, extra, m, dtype):
    cache, _ = make_cache(ck, 1, 1, [base], [extra], seed=4)
    n, q = base + extra, queries(m, G)
    clean, clean_lse = run(ck, cache, [m], q, dtype=dtype)
    inf, nan = float("inf"), float("nan")
    first = n - m
    pokes = [(first + m // 3, 5, inf), (first + m // 2, 5, -inf), (first + m // 4, 9, -inf), (n - 1, 70, nan), (first + m // 2, 127, inf), (first, 31, nan)]
    for row, col, value in pokes:
        poke(cache, 0, row, col, value, "v")
    out, lse = run(ck, cache, [m], q, dtype=dtype)
    # Finite or not: a part of a probability that is 0 or negative makes a NaN of an infinity that all queries of a block see.
    finite = torch.ones_like(clean, dtype=torch.bool)
    for row, col, _ in pokes:
        finite[max(0, row - first):, :, col] = False
    assert torch.equal(lse, clean_lse)
    assert torch.equal(torch.isfinite(out), finite)
    assert torch.equal(out[finite], clean[finite])  # bit for bit
    # a NaN in a key: the rows that see it, and no other
    for row, col, value in pokes:
        poke(cache, 0, row, col, 0.0, "v")
    ref, ref_lse = run(ck, cache, [m], q, dtype=dtype)
    poke(cache, 0, first + m // 2, 3, nan, "k")
    out, lse = run(ck, cache, [m], q, dtype=dtype)
    assert torch.equal(out[:m // 2], ref[:m // 2]) and torch.equal(lse[:m // 2], ref_lse[:m // 2])
    assert torch.isnan(out[m // 2:]).all() and torch.isnan(lse[m // 2:]).all()


def test_heads_before_tokens_orders_and_gaps(ck):
    B, Hkv, G = 4, 2, 3
    cache, rows = make_cache(ck, B, Hkv, [128, 256, 128, 0] * 2, [70] * 8, seed=8)
    n_new, start, n_tokens = [20, 1, 0, 33], [60, 41, 0, 5], 90
    x = queries(Hkv * G, n_tokens + 1)[:, 1:]
    q = x.transpose(0, 1)  # [n_tokens, Hq, D], the tokens of a head side by side
    assert q.stride(1) > q.stride(0)
    out, lse = run(ck, cache, n_new, q, start, n_tokens, sm_scale=0.2)
    check(out, lse, reference(rows, q, n_new, start, Hkv, float(np.float32(0.2))), 3.0)


def test_a_key_that_takes_everything(ck):
    """References that rise by far more than their slack, again and again, in both halves of a tile and from tile to tile."""
    for G, m, n in ((4, 6, 1000), (4, 64, 1000), (8, 300, 900)):
        cache, rows = make_cache(ck, 1, 1, [n], [0], seed=2)
        q = queries(m, G)
        k = rows[0][0]
        for j in range(0, n, 37):  # ever larger keys along the mean query
            v = (q.float().mean(dim=(0, 1)) * (0.05 * j)).bfloat16()
            cache.k_pool[int(cache.seg_off[0]) + j] = v
            k[j] = v.double()
        for dtype in (torch.float32, torch.bfloat16):
            out, lse = run(ck, cache, [m], q, dtype=dtype)
            check(out, lse, reference(rows, q, [m], [0], 1, D ** -0.5), 3.0)


def test_one_token_is_a_decode_step(ck):
    cache, _ = make_cache(ck, 3, 2, [640, 300, 128, 1000, 77, 512], [1, 200, 130, 0, 0, 65], seed=6)
    q = queries(3, 10)
    out, lse = run(ck, cache, [1, 1, 1], q)
    plan = ck.DecodePlan(cache, ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(cache, plan)
    want, want_lse = torch.zeros_like(out), torch.zeros_like(lse)
    ck.catekv_decode_attn(cache, q, plan, want, want_lse)
    # (decode attention carries its probabilities in 16 bits: 2^-17 of a value and 1e-6 in the norm)
    assert float((out - want).norm() / want.norm()) <= 1e-5 and float((lse - want_lse).abs().max()) <= 1e-5


def test_calls_repeat_bit_for_bit(ck):
    cache, _ = make_cache(ck, 2, 3, [700, 128, 384] * 2, [90] * 6, seed=3)
    for n_new in ([80, 3], [5, 2]):
        q = queries(sum(n_new), 12)
        for dtype in (torch.float32, torch.bfloat16):
            a, b = run(ck, cache, n_new, q, dtype=dtype), run(ck, cache, n_new, q, dtype=dtype)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_captured_step_follows_the_lists(ck):
    B, Hkv, G, n = 2, 2, 4, [3, 2]
    m = Model(ck, B, Hkv, [500] * 4, 30, 8, 11)
    ck.catekv_pages_reserve(m.cache, 60)
    chunk = ck.Chunk(n)
    q, k, v = queries(5, Hkv * G), queries(5, Hkv, 6), queries(5, Hkv, 7)
    out, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ws = ck.chunk_attn_workspace(m.cache, chunk, Hkv * G)
    ck.catekv_append_chunk(m.cache, chunk, k, v)
    ck.catekv_chunk_attn(m.cache, chunk, q, out, lse, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.catekv_append_chunk(m.cache, chunk, k, v)
        ck.catekv_chunk_attn(m.cache, chunk, q, out, lse, ws=ws)
    rows = lambda: [torch.cat([x, *[t[sum(n[:s // Hkv]):sum(n[:s // Hkv]) + n[s // Hkv], s % Hkv]] * reps]) for s in range(4) for x, t in zip(m.lists[s], (k, v))]
    for step in range(9):
        reps = step + 2
        k.copy_(queries(5, Hkv, 20 + step)), v.copy_(queries(5, Hkv, 40 + step)), q.copy_(queries(5, Hkv * G, 60 + step))
        g.replay()
        ck.catekv_cache_sync_lengths(m.cache)
        lens = m.cache.seg_len.tolist()
        assert lens == [500 + reps * n[s // Hkv] for s in range(4)]
        kv = [[x.double() for x in get_rows(m.cache, s, lens[s])] for s in range(4)]
        for s in range(4):
            b, h = divmod(s, Hkv)
            assert torch.equal(kv[s][0][-n[b]:], k[sum(n[:b]):sum(n[:b]) + n[b], h].double()) and torch.equal(kv[s][0][:500], m.lists[s][0].double())
        check(out, lse, reference(kv, q, n, [0, 3], Hkv, D ** -0.5), 3.0)
    assert ck.catekv_workspace_status(ws)["flags"] == 0


def test_a_replayed_append_stops_at_the_room_there_is(ck):
    """Rows for which a list has no room are dropped and not counted; nothing beside the list is written."""
    for n_new in (50, 100):  # one launch that counts, and two
        m = Model(ck, 1, 2, [200, 200], 8, 4, 5)
        ck.catekv_pages_reserve(m.cache, n_new)
        chunk = ck.Chunk([n_new])
        k, v = queries(n_new, 2), queries(n_new, 2, 9)
        room = [int(c) + 64 * int(p) for c, p in zip(m.cache.seg_cap, m.cache.pages.seg_pages)]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ck.catekv_append_chunk(m.cache, chunk, k, v)
        free = [p for p in range(8) if p not in set(m.cache.pages.table[0, :int(m.cache.pages.seg_pages[0])]) | set(m.cache.pages.table[1, :int(m.cache.pages.seg_pages[1])])]
        for i in range(4):
            g.replay()
        ck.catekv_cache_sync_lengths(m.cache)
        assert m.cache.seg_len.tolist() == [min(200 + 4 * n_new, r) for r in room]
        for s in range(2):
            got = get_rows(m.cache, s, int(m.cache.seg_len[s]))[0]
            want = torch.cat([m.lists[s][0], *[k[:, s]] * 4])[:got.shape[0]]
            assert torch.equal(got, want)
        for p in free:
            assert torch.isnan(m.cache.pages.k_ovf[p * 64:p * 64 + 64].float()).all()


def test_two_streams_at_once(ck):
    caches = [make_cache(ck, 2, 2, [1500, 900, 128, 3000], [40] * 4, seed=s) for s in (1, 2)]
    qs = [queries(70, 8, s) for s in (1, 2)]
    want = [run(ck, c, [60, 10], q) for (c, _), q in zip(caches, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    chunk = ck.Chunk([60, 10])
    wss = [ck.chunk_attn_workspace(c, chunk, 8) for c, _ in caches]
    outs = [(torch.zeros_like(a), torch.zeros_like(b)) for a, b in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                ck.catekv_chunk_attn(caches[i][0], chunk, qs[i], *outs[i], ws=wss[i])
    torch.cuda.synchronize()
    for (a, b), (c, d), ws in zip(outs, want, wss):
        assert torch.equal(a, c) and torch.equal(b, d) and ck.catekv_workspace_status(ws)["flags"] == 0


def test_waits_that_run_out_are_reported(ck):
    for n_new, dtype in ((3, torch.bfloat16), (100, torch.bfloat16), (100, torch.float32)):
        cache, rows = make_cache(ck, 1, 2, [640, 1500], [70, 70], seed=12)
        q = queries(n_new, 8)
        chunk = ck.Chunk([n_new])
        out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=dtype), torch.full(q.shape[:2], 3.0, device="cuda")
        ws = ck.chunk_attn_workspace(cache, chunk, 8)
        ck.catekv_test_expire_score_waits(1)
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
        with pytest.raises(ck.CatekvError) as e:
            ck.catekv_workspace_status(ws)
        assert e.value.code == ck.ERR_DEVICE
        st = ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)
        assert st["flags"] == ck.STATUS_WAIT_EXPIRED and st["kernel"] == 7
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)  # the context is whole, and the workspace too
        assert ck.catekv_workspace_status(ws)["flags"] == 0
        check(out, lse, reference(rows, q, [n_new], [0], 2, D ** -0.5), 3.0)


def test_rows_whose_byte_offset_passes_32_bits(ck):
    cache = ck.Cache(1, 2, [8_600_000, 300], 128)  # 2.2 GB a pool: the second list lies behind
    cache.set_lengths([250, 300])
    assert int(cache.seg_off[1]) * 256 > 2 ** 31
    x = queries(550, 2, 3)
    for s, n in ((0, 250), (1, 300)):
        o = int(cache.seg_off[s])
        cache.k_pool[o:o + n], cache.v_pool[o:o + n] = x[:n, 0], x[250:250 + n, 1]
    k, v = queries(70, 2, 8), queries(70, 2, 9)
    ck.catekv_append_chunk(cache, ck.Chunk([70]), k, v)
    rows = []
    for s, n in ((0, 320), (1, 370)):
        o = int(cache.seg_off[s])
        assert torch.equal(cache.k_pool[o + n - 70:o + n], k[:, s]) and torch.equal(cache.v_pool[o + n - 70:o + n], v[:, s])
        rows.append([cache.k_pool[o:o + n].double(), cache.v_pool[o:o + n].double()])
    q = queries(70, 8)
    out, lse = run(ck, cache, [70], q)
    check(out, lse, reference(rows, q, [70], [0], 2, D ** -0.5), 3.0)


def test_without_pages_and_without_lse(ck):
    cache = ck.Cache(2, 1, [200, 100], 64)
    m = [queries(200, 1, 3)[:, 0], queries(100, 1, 4)[:, 0]]
    for s in range(2):
        o = int(cache.seg_off[s])
        cache.k_pool[o:o + m[s].shape[0]], cache.v_pool[o:o + m[s].shape[0]] = m[s], m[s]
    cache.set_lengths([200, 100])
    q = queries(7, 5)
    want, _ = run(ck, cache, [4, 3], q)
    out = torch.zeros_like(want)
    ck.catekv_chunk_attn(cache, ck.Chunk([4, 3]), q, out)
    assert torch.equal(out, want)
    ck.catekv_truncate(cache, [150, 1000])
    assert cache.seg_len.tolist() == cache.seg_len_dev.tolist() == [50, 0]
    ck.catekv_append_chunk(cache, ck.Chunk([0, 5]), queries(5, 1), queries(5, 1))
    assert cache.seg_len.tolist() == cache.seg_len_dev.tolist() == [50, 5]
    out, lse = run(ck, cache, [0, 5], q[:5])
    o = int(cache.seg_off[1])
    rows = [[cache.k_pool[:50].double(), cache.v_pool[:50].double()], [cache.k_pool[o:o + 5].double(), cache.v_pool[o:o + 5].double()]]
    check(out, lse, reference(rows, q[:5], [0, 5], [0, 0], 1, D ** -0.5), 3.0)


def test_many_orders_in_one_fork(ck):
    """More orders than one launch's arguments hold, and parents that are replaced themselves."""
    B, Hkv = 96, 8
    m = Model(ck, B, Hkv, [130] * (B * Hkv), 12 * B * Hkv, 12, 1)
    ck.catekv_pages_reserve(m.cache, 300)
    m.append([300 if b % 2 else 17 for b in range(B)])
    m.fork([(b * 7 + 1) % B for b in range(B)])
    m.verify()
    m.truncate([b % 5 * 60 for b in range(B)])
    m.verify()
    assert ck.catekv_pages_compact(m.cache) == m.verify()


def test_a_pool_of_more_than_65536_pages(ck):
    m = Model(ck, 1, 1, [0], 65600, 8, 2)
    for i, page in enumerate((65599, 3, 65536, 65535)):
        m.cache.pages.table[0, i] = page
    m.cache.pages.seg_pages[0] = 4
    m.cache.pages.struct.next_free, m.cache.pages.struct.released = 65600, 65596
    m.cache.pages.table_dev.copy_(torch.from_numpy(m.cache.pages.table))
    m.append([250])
    m.verify()
    assert ck.catekv_pages_compact(m.cache) == 4
    assert sorted(m.cache.pages.table[0, :4].tolist()) == [0, 1, 2, 3] and m.cache.pages.table[0, 1] == 3  # the lowest goes to the first free place
    assert m.cache.pages.table[0, [3, 2, 0]].tolist() == [0, 1, 2]
    m.verify()


def test_a_call_that_is_refused_changes_nothing(ck):
    m = Model(ck, 2, 1, [100, 100], 2, 3, 4)
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_pages_reserve(m.cache, 100)  # one page each is there, two are wanted
    assert e.value.code == ck.ERR_CAPACITY
    m.fork([0, 0])
    with pytest.raises(ck.CatekvError) as e:
        m.append([65, 0])
    assert e.value.code == ck.ERR_CAPACITY
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_chunk_attn(m.cache, ck.Chunk([101, 0]), queries(101, 4), torch.zeros(101, 4, D, device="cuda"))
    assert e.value.code == ck.ERR_INVALID_ARG
    m.verify()


@pytest.mark.parametrize("G,m", [(4, 5), (4, 100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_queries_that_see_nothing(ck, G, m, dtype):
    """A replayed call may find a list with fewer rows than the chunk has tokens: the first queries then see none of them."""
    for n in (0, 1, 3, 64):
        cache, rows = make_cache(ck, 1, 2, [200, 256], [0, 0], seed=9)
        cache.seg_len_dev.copy_(torch.tensor([n, 256], dtype=torch.int32))
        for pool in (cache.k_pool, cache.v_pool):
            pool[int(cache.seg_off[0]) + n:int(cache.seg_off[0]) + 200] = float("nan")
        q = queries(m, 2 * G)
        out, lse = run(ck, cache, [m], q, dtype=dtype)
        none = max(0, m - n)
        assert (out[:none, :G] == 0).all() and (lse[:none, :G] == float("-inf")).all()
        # (the other list's results too: where blocks are cut between CTAs, and so the order of the sums, goes by all lists' lengths)
        for h, length, kv in ((0, n, [x[:n] for x in rows[0]]), (1, 256, rows[1])):
            at = slice(h * G, (h + 1) * G)
            for i in range(none if h == 0 else 0, m):
                see = length - m + i + 1
                z = q[i, at].double() @ kv[0][:see].T * D ** -0.5
                assert float((lse[i, at].double() - torch.logsumexp(z, 1)).abs().max()) <= 1e-5
                p = torch.softmax(z, 1)
                o = p @ kv[1][:see]
                # a bf16 result and its probabilities are off by half a step each (2^-8), an fp32 result by 1e-5 of the row
                tol = 4e-5 if dtype == torch.float32 else 2.0 ** -8
                bound = tol * (o.abs() + p @ kv[1][:see].abs()) + 4e-5 * o.abs().amax()
                assert ((out[i, at].double() - o).abs() <= bound).all()


def test_the_chunk_steps_of_the_readme(ck):
    import os
    import re
    import paper_2608_30295_b200 as pkg
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        block, = re.findall(r"```py\n(.*?)```", f.read(), flags=re.S)
    cache = ck.Cache(3, 2, [300] * 6, 0)
    cache.k_pool.normal_(), cache.v_pool.normal_()
    cache.set_lengths([300] * 6)
    names = {"ck": pkg, "cache": cache, "n_pages": 40, "max_pages": 6, "n_new": [5, 1, 80], "Hq": 8, "k_new": queries(86, 2), "v_new": queries(86, 2, 9),
             "q": queries(86, 8), "out": torch.full((86, 8, D), float("nan"), device="cuda"), "lse": torch.zeros(86, 8, device="cuda"),
             "n_rejected": [3, 0, 20], "parent": [0, 1, 1]}
    exec(block, names)
    assert torch.isfinite(names["out"]).all()
    assert cache.seg_len.tolist() == cache.seg_len_dev.tolist() == [302, 302, 301, 301, 301, 301]
    assert names["pages_in_use"] == int(cache.pages.seg_pages.sum())
