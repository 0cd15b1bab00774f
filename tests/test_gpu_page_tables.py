"""What the page calls leave in the host's and the device's tables, and when they may be captured."""
import numpy as np
import numpy as np
import pytest
import torch

from test_gpu_chunk import D
from test_gpu_pages import Model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def state(m):
    c, p = m.cache, m.cache.pages
    return [x.tolist() for x in (c.seg_off, c.seg_cap, c.seg_len, p.table, p.seg_pages)] + [p.struct.next_free, p.struct.released]


def test_pages_are_not_handed_out_or_moved_in_a_capture(ck):
    """The orders travel in the launch: a replay would name pages that other lists may hold by then."""
    m = Model(ck, 2, 1, [100, 100], 10, 4, 2)
    ck.catekv_pages_reserve(m.cache, 100)
    m.append([100, 100])
    m.truncate([100, 0])  # the second list's pages lie behind free ones
    before, codes = state(m), []
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for call in (lambda: ck.catekv_pages_reserve(m.cache, 100), lambda: ck.catekv_pages_compact(m.cache)):
            try:
                call()
            except ck.CatekvError as e:
                codes.append(e.code)
        ck.catekv_pages_reserve(m.cache, 10)  # there is room: nothing is handed out
    assert codes == [ck.ERR_UNSUPPORTED] * 2 and state(m) == before
    m.verify()
    assert ck.catekv_pages_compact(m.cache) == 2
    ck.catekv_pages_reserve(m.cache, 100)
    m.append([100, 100])
    m.verify()


def check_tables(m):
    """Host and device agree on every entry; those behind the pages in force are -1, or name a page that is free and no other list's row names."""
    p = m.cache.pages
    torch.cuda.synchronize()
    assert p.table_dev.tolist() == p.table.tolist()
    used = {int(x) for s in range(m.S) for x in p.table[s, :int(p.seg_pages[s])]}
    behind = [int(x) for s in range(m.S) for x in p.table[s, int(p.seg_pages[s]):] if x >= 0]
    assert len(set(behind)) == len(behind) and not used & set(behind)


def test_tables_name_no_page_of_another_list(ck):
    m = Model(ck, 4, 2, [300] * 8, 80, 12, 5)
    for step in (lambda: ck.catekv_pages_reserve(m.cache, 400), lambda: m.append([400, 10, 130, 0]), lambda: m.truncate([250, 0, 1, 300]),
                 lambda: m.fork([0, 0, 2, 2]), lambda: ck.catekv_pages_reserve(m.cache, 70), lambda: m.append([3, 70, 64, 1]), lambda: m.fork([2, 3, 0, 1]),
                 lambda: ck.catekv_pages_compact(m.cache), lambda: m.truncate([5000, 200, 130, 129]), lambda: m.fork([3, 1, 1, 3])):
        step()
        m.verify()
        check_tables(m)


def given_back(ck, n_new, append):
    """A captured append whose list 0 has room for 20 rows more and whose former pages list 1 has got."""
    m = Model(ck, 2, 1, [128, 128], 8, 4, 1)
    ck.catekv_pages_reserve(m.cache, n_new)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        append(m.cache)
    ck.catekv_cache_sync_lengths(m.cache)  # (nothing has run)
    mine = m.cache.pages.table[0, :int(m.cache.pages.seg_pages[0])].tolist()
    m.append([n_new, 64 * len(mine)])
    m.truncate([n_new + 20, 0])
    ck.catekv_pages_reserve(m.cache, 20)
    m.append([0, 20])
    assert m.cache.pages.seg_pages.tolist() == [0, len(mine) + 1] and m.cache.pages.table[1, len(mine)] == mine[0]
    m.verify()
    return m, g


@pytest.mark.parametrize("n_new", [30, 100])  # one launch, and two
def test_a_replayed_append_does_not_follow_a_page_that_was_given_back(ck, n_new):
    k, v = (torch.randn(n_new, 1, D, device="cuda").bfloat16() for _ in range(2))
    m, g = given_back(ck, n_new, lambda cache: ck.catekv_append_chunk(cache, ck.Chunk([n_new, 0]), k, v))
    for _ in range(2):
        g.replay()
    ck.catekv_cache_sync_lengths(m.cache)
    assert m.cache.seg_len.tolist() == [128, m.lists[1][0].shape[0]]
    m.lists[0] = [torch.cat([x, new[:20, 0]]) for x, new in zip(m.lists[0], (k, v))]
    m.verify()


@pytest.mark.parametrize("steps", [25, 60])  # the second one: list 1 has no room left either
def test_a_replayed_token_does_not_follow_a_page_that_was_given_back(ck, steps):
    k, v = (torch.randn(2, 1, D, device="cuda").bfloat16() for _ in range(2))
    m, g = given_back(ck, 30, lambda cache: ck.catekv_append(cache, k, v))
    for _ in range(steps):
        g.replay()
    ck.catekv_cache_sync_lengths(m.cache)
    for s, n in ((0, 20), (1, min(steps, 44))):
        m.lists[s] = [torch.cat([x, *[new[s]] * n]) for x, new in zip(m.lists[s], (k, v))]
    m.verify()


def test_a_plan_made_before_rows_were_taken_back(ck):
    """It knows rows in pages that the list has given back: they are left out, whoever has the pages now."""
    G = 4
    m = Model(ck, 3, 1, [100] * 3, 14, 12, 3)
    ck.catekv_pages_reserve_each(m.cache, [300, 300, 0])
    m.append([300, 300, 0])
    plan = ck.DecodePlan(m.cache, 7)
    ck.catekv_decode_plan(m.cache, plan)
    q = torch.randn(3, G, D, device="cuda").bfloat16()
    out, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    odd = torch.full((400, 1, D), float("inf"), device="cuda", dtype=torch.bfloat16)
    for drop, add in (([250, 0, 0], [0, 0, 150]), ([0, 20, 0], [0, 0, 60]), ([90, 200, 0], [0, 0, 250]), ([0, 0, 0], [7, 5, 0])):
        m.truncate(drop)
        check_tables(m)
        ck.catekv_pages_reserve_each(m.cache, add)
        check_tables(m)
        if add[2]:  # the third sequence gets the pages, and rows of infinities
            ck.catekv_append_chunk(m.cache, ck.Chunk(add), odd[:add[2]], odd[:add[2]])
            m.lists[2] = [torch.cat([x, odd[:add[2], 0]]) for x in m.lists[2]]
        else:
            m.append(add)
        m.verify()
        ck.catekv_decode_attn(m.cache, q, plan, out, lse)
        for b in range(2):
            kk, vv = (x.double() for x in m.lists[b])
            z = q[b].double() @ kk.T * D ** -0.5
            o = torch.softmax(z, 1) @ vv
            assert float((out[b].double() - o).norm() / o.norm()) <= 1e-5
            assert float((lse[b].double() - torch.logsumexp(z, 1)).abs().max()) <= 1e-5


def test_drafts_keep_the_tables_entries(ck):
    """Pages given back and reserved again by the same lists: the same entries, and no order for the device in between."""
    m = Model(ck, 3, 2, [200] * 6, 60, 8, 5)
    ck.catekv_pages_reserve(m.cache, 150)
    first = m.cache.pages.table.copy()
    for _ in range(3):
        m.append([150, 100, 3])
        m.truncate([150, 100, 3])
        torch.cuda.synchronize()
        assert (m.cache.pages.table == first).all() and m.cache.pages.table_dev.tolist() == first.tolist()
        m.verify()
        check_tables(m)
        ck.catekv_pages_reserve(m.cache, 150)


def test_many_sequences_leave_shared_rows_in_turn(ck):
    """Who still reads a segment's rows behind a new end goes by the lists before it in the same call as they are left, and by those after it as they were."""
    B = 24
    m = Model(ck, B, 2, [700] * (B * 2), 40 * B, 24, 6)
    m.fork([b % 3 for b in range(B)])
    m.verify()
    for drop in ([60] + [0] * 23, [300] * 4 + [100] * 4 + [0] * 16, [0] * 12 + [400] * 6 + [5] * 6, [130] * 24, [0, 10, 500] * 8, [5000] * 20 + [1] * 4):
        m.truncate(drop)
        m.verify()
        ck.catekv_pages_reserve(m.cache, 70)
        m.append([70 - 3 * b if b % 4 else 0 for b in range(B)])
        m.verify()
        check_tables(m)


def test_rows_taken_back_and_appended_anew_under_one_plan(ck):
    """The plan knows the places of the new rows: attention that follows the append at once must not read them before they are written."""
    B, Hkv, G = 8, 4, 4
    m = Model(ck, B, Hkv, [500] * (B * Hkv), 200, 8, 3)
    ck.catekv_pages_reserve(m.cache, 200)
    m.append([120] * B)
    plan = ck.DecodePlan(m.cache, ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(m.cache, plan)
    out, lse = torch.zeros((B, Hkv * G, D), device="cuda"), torch.zeros((B, Hkv * G), device="cuda")
    for step in range(12):
        n = 100 + 3 * step
        m.truncate([n] * B)
        ck.catekv_pages_reserve(m.cache, n)
        q = torch.randn(B, Hkv * G, D, device="cuda").bfloat16()
        m.append([n] * B)
        ck.catekv_decode_attn(m.cache, q, plan, out, lse)
        for s in range(m.S):
            b, h = divmod(s, Hkv)
            k, v = (x.double() for x in m.lists[s])
            z = q[b, h * G:h * G + G].double() @ k.T * D ** -0.5
            o = torch.softmax(z, 1) @ v
            assert float((out[b, h * G:h * G + G].double() - o).norm() / o.norm()) <= 1e-5
            assert float((lse[b, h * G:h * G + G].double() - torch.logsumexp(z, 1)).abs().max()) <= 1e-5


@pytest.mark.parametrize("seed", range(4))
def test_next_free_follows_the_pages_in_use(ck, seed):
    """Pages are handed out from next_free on while none below it is free: it lies behind every page in use, and after a call that counts them right behind."""
    rng = np.random.default_rng(100 + seed)
    B, Hkv = int(rng.integers(2, 6)), int(rng.integers(1, 4))
    m = Model(ck, B, Hkv, [200] * (B * Hkv), 40 * B * Hkv, 60, seed)
    p = m.cache.pages
    for _ in range(20):
        what, counted = rng.integers(0, 5), False
        if what <= 1 and max(x[0].shape[0] for x in m.lists) < 2000:
            n_new = [int(rng.choice([0, 1, 64, 100])) for _ in range(B)]
            ck.catekv_pages_reserve(m.cache, max(n_new))
            m.append(n_new)
        elif what == 2:
            parent = [int(rng.integers(0, B)) for _ in range(B)]
            counted = parent != list(range(B))
            m.fork(parent)
        elif what == 3:
            drop = [int(rng.choice([0, 1, 64, 130, 5000])) for _ in range(B)]
            counted = any(drop)
            m.truncate(drop)
        else:
            counted = ck.catekv_pages_compact(m.cache) >= 0
        m.verify()
        used = {int(x) for s in range(m.S) for x in p.table[s, :int(p.seg_pages[s])]}
        top = max(used) + 1 if used else 0
        assert p.struct.next_free == top if counted else p.struct.next_free >= top
        assert p.struct.released == p.struct.next_free - len(used)
        assert p.struct.next_free <= p.struct.n_pages


def test_a_mixed_batch_gets_the_pages_it_needs(ck):
    """A piece of a prompt beside sequences that decode: pages for the piece in its sequence's lists alone."""
    B, Hkv = 8, 2
    m = Model(ck, B, Hkv, [128] * (B * Hkv), 40, 12, 4)
    n_new = [0, 1, 600, 1, 0, 1, 70, 1]
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_pages_reserve(m.cache, max(n_new))  # 10 pages for each of the 16 lists
    assert e.value.code == ck.ERR_CAPACITY
    ck.catekv_pages_reserve_each(m.cache, n_new)
    assert m.cache.pages.seg_pages.tolist() == [-(-n // 64) for n in n_new for _ in range(Hkv)]
    m.append(n_new)
    m.verify()
    check_tables(m)
    ck.catekv_pages_reserve_each(m.cache, [0] * B)  # nothing to do
    m.truncate([0, 0, 300, 0, 0, 0, 70, 0])
    ck.catekv_pages_reserve_each(m.cache, [300, 0, 0, 0, 100, 0, 0, 0])
    m.append([300, 63, 20, 0, 100, 0, 0, 0])
    m.verify()
    check_tables(m)
    before = state(m)
    for n in ([1] * (B - 1), [-1] + [0] * (B - 1), None):
        with pytest.raises((ck.CatekvError, TypeError)):
            ck.catekv_pages_reserve_each(m.cache, n)
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_pages_reserve_each(m.cache, [5000] + [0] * (B - 1))  # more than a table row holds
    assert e.value.code == ck.ERR_CAPACITY and state(m) == before
