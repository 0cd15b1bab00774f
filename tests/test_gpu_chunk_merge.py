"""Chunk attention where blocks of queries are cut into few pieces or many, and where there are more lists than a CTA has threads; against the
definition in 64 bits, with the tolerances of the other tests of it."""
import pytest
import torch

from test_gpu_chunk import D, check, make_cache, reference
from test_gpu_chunk_edges import poke, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


CASES = [
    # B, Hkv, G, base, extra, n_new
    (1, 1, 8, [20000], [0], [1]),          # one block, as many pieces as CTAs
    (1, 1, 8, [20000], [200], [16]),
    (1, 1, 4, [15000], [0], [64]),         # the same with two M tiles
    (1, 2, 8, [9000], [0], [12]),          # some 70 pieces
    (1, 3, 4, [2000], [70], [4]),          # some 17
    (2, 8, 7, [1500], [100], [18, 3]),     # a few
    (120, 8, 2, [128, 0, 256], [5], [1, 2, 0, 3]),   # 960 lists
    (500, 2, 1, [0, 128], [3], [1, 0, 0, 2, 0]),     # 1000 lists, most of them without a query
    (45, 8, 4, [384, 128, 900], [3], [0, 0, 0, 0, 70, 1, 0, 0, 0]),  # 360: one round of threads with bf16 results, two with fp32
]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_pieces_and_many_lists(ck, case, out_dtype):
    B, Hkv, G, base, extra, n_new = case
    S = B * Hkv
    base, extra, n_new = (base * S)[:S], (extra * S)[:S], (n_new * B)[:B]
    extra = [max(e, n_new[s // Hkv] - b) for s, (b, e) in enumerate(zip(base, extra))]
    cache, rows = make_cache(ck, B, Hkv, base, extra, seed=S)
    q = queries(sum(n_new), Hkv * G)
    out, lse = run(ck, cache, n_new, q, dtype=out_dtype)
    check(out, lse, reference(rows, q, n_new, [sum(n_new[:b]) for b in range(B)], Hkv, D ** -0.5), 3.0)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("G,n_new", [(4, [1, 2]), (4, [80, 3])])
def test_lists_that_were_whole_when_the_call_was_captured(ck, G, n_new, out_dtype):
    """The host chooses the number of CTAs from short lists; replayed over long ones, the blocks are cut all the same, or one CTA has them all."""
    B, Hkv = 2, 2
    cache, rows = make_cache(ck, B, Hkv, [6000, 100, 2500, 128], [90, 0, 0, 200], seed=4)
    long = [k.shape[0] for k, _ in rows]
    T = sum(n_new)
    q, start = queries(T, Hkv * G), [0, n_new[0]]
    out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=out_dtype), torch.full(q.shape[:2], 3.0, device="cuda")
    chunk = ck.Chunk(n_new)
    ws = ck.chunk_attn_workspace(cache, chunk, Hkv * G)
    short = [90, 80, 85, 81]
    cache.set_lengths(short)
    ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    for lens in (long, short, [6000, 90, 90, 300], long):
        cache.set_lengths(lens)
        g.replay()
        now = [(k[:n], v[:n]) for (k, v), n in zip(rows, lens)]
        check(out, lse, reference(now, q, n_new, start, Hkv, D ** -0.5), 3.0)
    assert ck.catekv_workspace_status(ws)["flags"] == 0


@pytest.mark.parametrize("n_new", [1, 40])
def test_pieces_that_see_nothing_or_meet_an_infinity(ck, n_new):
    """A list in many pieces: keys so far below the others that their pieces add nothing, one piece whose keys are all at -inf, and one infinity in V."""
    G = 4
    cache, rows = make_cache(ck, 1, 1, [9000], [0], seed=2)
    n = 9000
    q = queries(n_new, G)
    q[..., 0] = 1.0
    (k, v), = rows
    k = k.clone()
    for lo, hi, x in ((0, 3000, -6000.0), (4000, 4700, float("-inf"))):
        k[lo:hi, 0] = x
        off = int(cache.seg_off[0])
        cache.k_pool[off + lo:off + hi, 0] = x
    want = reference([(k, v)], q, [n_new], [0], 1, D ** -0.5)
    for dtype in (torch.float32, torch.bfloat16):
        out, lse = run(ck, cache, [n_new], q, dtype=dtype)
        check(out, lse, want, 3.0)
    poke(cache, 0, 100, 7, float("inf"), "v")  # its probability is 0, and 0 * inf is no number
    poke(cache, 0, 8000, 9, float("-inf"), "v")
    for dtype in (torch.float32, torch.bfloat16):
        out, _ = run(ck, cache, [n_new], q, dtype=dtype)
        bad = ~torch.isfinite(out)
        assert bad[..., 9].all() and not bad[..., :7].any() and not bad[..., 10:].any()


@pytest.mark.parametrize("G,n_new", [(4, [4, 0, 16, 1]), (7, [9, 2, 1, 9]), (1, [64, 1, 33, 32]), (8, [1, 1, 1, 1]), (3, [21, 20, 1, 0])])
def test_few_rows_over_long_lists(ck, G, n_new):
    """bf16 results, at most 64 query rows a block, more than 1776 tiles in all: the form whose low parts have rows of their own."""
    B, Hkv = 4, 8
    base = [9000, 8192, 7000 + 61, 10000] * 8
    cache, rows = make_cache(ck, B, Hkv, base, [70, 0, 5, 200] * 8, seed=G)
    q = queries(sum(n_new), Hkv * G)
    start = [sum(n_new[:b]) for b in range(B)]
    want = reference(rows, q, n_new, start, Hkv, D ** -0.5)
    out, lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    check(out, lse, want, 3.0)
    # the two parts of P carry 17 bits: what is left is the rounding of the result
    there = ~torch.isnan(want[1])
    w, g = want[0][there], out[there].double()
    assert ((g - w).abs() <= w.abs() * 2.0 ** -8 + 1e-5 * w.abs().amax(dim=-1, keepdim=True) * 4).all()
    again, lse2 = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_few_rows_over_long_lists_with_numbers_that_are_not_finite(ck):
    n_new, Hkv, G = [5, 3], 8, 4
    cache, rows = make_cache(ck, 2, Hkv, [16000] * 16, [40] * 16, seed=8)
    q = queries(8, Hkv * G)
    want = reference(rows, q, n_new, [0, 5], Hkv, D ** -0.5)
    n = 16040
    poke(cache, 0, n - 3, 11, float("inf"), "v")    # the third of five new rows: tokens 2, 3 and 4 see it
    poke(cache, 9, n - 1, 12, float("nan"), "k")    # list (1, 1): the last token alone
    poke(cache, 2, 77, 5, float("-inf"), "v")       # an old row: every token of the list
    out, lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    bad = ~torch.isfinite(out)
    assert bad[2:5, 0:G, 11].all() and bad[7, G:2 * G].all() and bad[:5, 2 * G:3 * G, 5].all()
    bad[2:5, 0:G, 11] = bad[7, G:2 * G] = bad[:5, 2 * G:3 * G, 5] = False
    assert not bad.any()
    fine = torch.isfinite(out)
    tol = (want[0].abs() + want[2]) * 2.0 ** -8 + 1e-5 * want[0].abs().amax(dim=-1, keepdim=True) * 4
    assert ((out.double() - want[0]).abs() <= tol)[fine].all()
