"""Pages of a cache: random sequences of appends, forks, truncations and compactions against lists kept in plain Python, row by row, and decode
and chunk attention over what they leave."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import D, check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def device_rows(cache, s, pool, ovf):
    """The rows of list s by the device's own tables."""
    n, cap, off = (int(t[s]) for t in (cache.seg_len_dev, cache.seg_cap_dev, cache.seg_off_dev))
    out = [pool[off:off + min(n, cap)]]
    for p in range(-(-max(0, n - cap) // 64)):
        pg = int(cache.pages.table_dev[s, p])
        assert 0 <= pg < cache.pages.struct.n_pages
        out.append(ovf[pg * 64:pg * 64 + min(64, n - cap - 64 * p)])
    return torch.cat(out)


class Model:
    """Lists as plain tensors, and a cache that has to hold the same."""

    def __init__(self, ck, B, Hkv, len0, n_pages, max_pages, seed):
        self.ck, self.B, self.Hkv, self.S = ck, B, Hkv, B * Hkv
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cache = ck.Cache(B, Hkv, [0 if n is None else n for n in len0], 0)
        self.cache.attach_pages(n_pages, max_pages)
        for t in (self.cache.k_pool, self.cache.v_pool, self.cache.pages.k_ovf, self.cache.pages.v_ovf):
            t.fill_(float("nan"))
        self.lists = [[torch.zeros(0, D, device="cuda", dtype=torch.bfloat16)] * 2 for _ in range(self.S)]
        start = [int(n or 0) for n in len0]
        per = [max(start[b * Hkv:(b + 1) * Hkv]) for b in range(B)]
        assert all(n == per[i // Hkv] for i, n in enumerate(start))
        self.append(per)

    def append(self, n_new, one=False):
        k, v = (torch.randn(max(sum(n_new), 1), self.Hkv, D, generator=self.gen, device="cuda").bfloat16() for _ in range(2))
        if one:  # the decode step's append
            self.ck.catekv_append(self.cache, k.reshape(self.B, self.Hkv, D), v.reshape(self.B, self.Hkv, D))
        else:
            chunk = self.ck.Chunk(n_new, n_tokens=k.shape[0])
            self.ck.catekv_append_chunk(self.cache, chunk, k, v)
        at = 0
        for b, n in enumerate(n_new):
            for h in range(self.Hkv):
                s = b * self.Hkv + h
                self.lists[s] = [torch.cat([x, new[at:at + n, h]]) for x, new in zip(self.lists[s], (k, v))]
            at += n

    def fork(self, parent):
        self.ck.catekv_fork(self.cache, parent)
        old = list(self.lists)
        for b, p in enumerate(parent):
            for h in range(self.Hkv):
                self.lists[b * self.Hkv + h] = old[p * self.Hkv + h]

    def truncate(self, drop):
        self.ck.catekv_truncate(self.cache, drop)
        for s in range(self.S):
            self.lists[s] = [x[:max(0, x.shape[0] - drop[s // self.Hkv])] for x in self.lists[s]]

    def verify(self):
        c, p = self.cache, self.cache.pages
        torch.cuda.synchronize()
        assert c.seg_len.tolist() == c.seg_len_dev.tolist() == [x[0].shape[0] for x in self.lists]
        assert c.seg_off.tolist() == c.seg_off_dev.tolist() and c.seg_cap.tolist() == c.seg_cap_dev.tolist()
        used, table = set(), p.table_dev.cpu().numpy()
        for s in range(self.S):
            n = int(p.seg_pages[s])
            assert np.array_equal(p.table[s, :n], table[s, :n])
            assert int(c.seg_len[s]) <= int(c.seg_cap[s]) + 64 * n
            used |= set(p.table[s, :n].tolist())
            for x, pool, ovf in zip(self.lists[s], (c.k_pool, c.v_pool), (p.k_ovf, p.v_ovf)):
                assert torch.equal(device_rows(c, s, pool, ovf), x), s
        assert p.struct.next_free == (max(used) + 1 if used else 0) or p.struct.released == p.struct.next_free - len(used)
        assert p.struct.released == p.struct.next_free - len(used)
        return len(used)


@pytest.mark.parametrize("seed", range(12))
def test_random_walks(ck, seed):
    rng = np.random.default_rng(seed)
    B, Hkv = int(rng.integers(1, 6)), int(rng.integers(1, 4))
    per = [int(rng.choice([0, 1, 63, 64, 127, 128, 129, 300])) for _ in range(B)]
    m = Model(ck, B, Hkv, [per[s // Hkv] for s in range(B * Hkv)], 40 * B * Hkv, 60, seed)
    m.verify()
    for _ in range(25):
        what = rng.integers(0, 6)
        longest = max(x[0].shape[0] for x in m.lists)
        if what <= 1 and longest < 2500:
            n_new = [int(rng.choice([0, 1, 5, 64, 100, 200])) for _ in range(B)]
            ck.catekv_pages_reserve(m.cache, max(n_new))
            m.append(n_new)
        elif what == 2 and longest < 2500:
            ck.catekv_pages_reserve(m.cache, 1)
            m.append([1] * B, one=True)
        elif what == 3:
            m.fork([int(rng.integers(0, B)) if rng.random() < 0.6 else b for b in range(B)])
        elif what == 4:
            m.truncate([int(rng.choice([0, 0, 1, 3, 64, 130, 5000])) for _ in range(B)])
        else:
            n = ck.catekv_pages_compact(m.cache)
            assert n == m.verify() == m.cache.pages.struct.next_free and m.cache.pages.struct.released == 0
        m.verify()


def test_swapped_beams_and_equal_parents(ck):
    m = Model(ck, 4, 2, [200] * 8, 100, 20, 3)
    ck.catekv_pages_reserve(m.cache, 100)
    m.append([10, 70, 100, 0])
    m.fork([1, 0, 3, 2])
    m.verify()
    m.fork([1, 1, 1, 1])
    m.verify()
    ck.catekv_pages_reserve(m.cache, 60)
    m.append([60, 1, 0, 33])  # they grow apart
    m.verify()
    m.truncate([61, 2, 3, 40])  # into rows that are shared
    m.verify()
    m.truncate([5000, 0, 5000, 0])
    m.verify()
    ck.catekv_pages_reserve(m.cache, 10)
    m.append([10, 10, 10, 10])
    m.verify()


def test_drafted_tokens_are_verified_and_taken_back(ck):
    """A run as it is used: fork, drafts appended, attended to, partly taken back, a decode step over what is left."""
    B, Hkv, G = 3, 2, 4
    m = Model(ck, B, Hkv, [500] * 6, 60, 16, 7)
    m.fork([0, 0, 2])
    g = torch.Generator(device="cuda").manual_seed(1)
    for n_new, accepted in (([4, 3, 1], [1, 3, 0]), ([40, 2, 0], [40, 0, 0]), ([1, 1, 1], [1, 1, 1])):
        ck.catekv_pages_reserve(m.cache, max(n_new))
        m.append(n_new)
        chunk = ck.Chunk(n_new)
        q = torch.randn(sum(n_new), Hkv * G, D, generator=g, device="cuda").bfloat16()
        out, lse = torch.full(q.shape, 3.0, device="cuda"), torch.full(q.shape[:2], 3.0, device="cuda")
        assert ck.catekv_workspace_status(ck.catekv_chunk_attn(m.cache, chunk, q, out, lse))["flags"] == 0
        rows = [[x.double() for x in kv] for kv in m.lists]
        start = [sum(n_new[:b]) for b in range(B)]
        check(out, lse, reference(rows, q, n_new, start, Hkv, D ** -0.5), 3.0)
        m.truncate([n - a for n, a in zip(n_new, accepted)])
        m.verify()
    ck.catekv_pages_compact(m.cache)
    plan = ck.DecodePlan(m.cache, ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(m.cache, plan)
    q = torch.randn(B, Hkv * G, D, generator=g, device="cuda").bfloat16()
    out, lse = torch.zeros(q.shape, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ck.catekv_decode_attn(m.cache, q, plan, out, lse)
    rows = [[x.double() for x in kv] for kv in m.lists]
    check(out, lse, reference(rows, q, [1] * B, list(range(B)), Hkv, D ** -0.5), 3.0)
    m.fork([1, 1, 1])
    with pytest.raises(ck.CatekvError) as e:  # a plan holds the places of the lists that the fork has changed
        ck.catekv_decode_attn(m.cache, q, plan, out, lse)
    assert e.value.code == ck.ERR_INVALID_ARG


def test_released_pages_are_given_out_again(ck):
    m = Model(ck, 2, 1, [128, 128], 6, 6, 1)
    ck.catekv_pages_reserve(m.cache, 192)  # all six pages
    m.append([192, 192])
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_pages_reserve(m.cache, 1)
    assert e.value.code == ck.ERR_CAPACITY
    m.truncate([100, 0])
    assert m.verify() == 5 and m.cache.pages.table[0, :2].tolist() == [0, 1]
    with pytest.raises(ck.CatekvError):
        ck.catekv_pages_reserve(m.cache, 36 + 1)  # list 1 would need a second page more
    m.truncate([0, 64])
    ck.catekv_pages_reserve(m.cache, 64)
    m.append([64, 64])
    assert m.verify() == 6


def test_unshared_copy_of_a_fork(ck):
    m = Model(ck, 3, 2, [300] * 6, 30, 8, 9)
    m.fork([0, 0, 0])
    ck.catekv_pages_reserve(m.cache, 20)
    m.append([3, 20, 7])
    dst = ck.catekv_cache_regrow(m.cache, 64)
    for s in range(6):
        n, o = int(dst.seg_len[s]), int(dst.seg_off[s])
        assert torch.equal(dst.k_pool[o:o + n], m.lists[s][0]) and torch.equal(dst.v_pool[o:o + n], m.lists[s][1])


def test_host_tables_cannot_be_captured(ck):
    m = Model(ck, 2, 1, [100, 100], 10, 4, 2)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    codes = []
    with torch.cuda.graph(g):
        for call in (lambda: ck.catekv_fork(m.cache, [0, 0]), lambda: ck.catekv_truncate(m.cache, [1, 0])):
            try:
                call()
            except ck.CatekvError as e:
                codes.append(e.code)
    assert codes == [ck.ERR_UNSUPPORTED] * 2
    m.verify()
