"""bf16 results of chunk attention are the exact ones rounded once: in every form of the kernel the probabilities carry 17 bits.

Tolerance, element by element.  The result's rounding: half a step, 2^-8 of the value at most.  A probability in two bf16 parts is off by 2^-9 of 2^-9
of itself, 2^-18: 2^-18 sum p |v|.  fp32 logits, sums and accumulators: 4e-5 of the row's largest element, as in the other tests of it."""
import pytest
import torch

from test_gpu_chunk import D, make_cache, reference
from test_gpu_chunk_edges import poke, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def check_rounded_once(out, lse, want):
    w, want_lse, mass = want
    there = ~torch.isnan(want_lse)
    assert (out[~there] == 3.0).all() and (lse[~there] == 3.0).all()
    w, g, mass = w[there], out[there].double(), mass[there]
    tol = w.abs() * 2.0 ** -8 + mass * 2.0 ** -18 + 4e-5 * w.abs().amax(dim=-1, keepdim=True)
    assert ((g - w).abs() <= tol).all(), float(((g - w).abs() - tol).max())
    assert float((lse[there].double() - want_lse[there]).abs().max()) <= 1e-5 * max(1.0, float(want_lse[there].abs().max()))


def starts(n_new):
    return [sum(n_new[:b]) for b in range(len(n_new))]


CASES = [
    # B, Hkv, G, base, extra, n_new
    (1, 1, 4, [4000], [0], [33]),            # a block and a little
    (1, 1, 4, [4000], [0], [300]),
    (2, 4, 4, [3000, 2944, 1000, 384], [0], [300, 41]),
    (1, 1, 1, [0], [700], [700]),
    (3, 2, 7, [128, 640], [300, 41], [100, 1, 33]),
    (2, 2, 8, [1500], [70], [16, 5]),        # at most 128 rows
    (4, 2, 5, [2000, 300], [0], [1, 2, 25, 0]),
    # more K and V than L2 holds, and queries for two M tiles a block
    (16, 8, 4, [2048], [60], [64]),
    (16, 8, 7, [2176, 2048], [31], [36, 30]),
    (15, 8, 1, [2816, 2560, 2600], [100, 0, 3], [256, 200, 0, 255, 129]),
    (16, 8, 3, [2000], [200], [84, 85, 1, 80]),
    (4, 8, 8, [9000], [5], [100, 31, 64, 130]),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_bf16_results_are_rounded_once(ck, case):
    B, Hkv, G, base, extra, n_new = case
    S = B * Hkv
    base, extra, n_new = (base * S)[:S], (extra * S)[:S], (n_new * B)[:B]
    cache, rows = make_cache(ck, B, Hkv, base, extra, seed=S + G)
    q = queries(sum(n_new), Hkv * G, G)
    out, lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    check_rounded_once(out, lse, reference(rows, q, n_new, starts(n_new), Hkv, D ** -0.5))


def two_tiles(ck, B=16, Hkv=8, G=4, m=64, extra=60):
    """A cache whose K and V are 140 MB, and queries of two full M tiles for every list."""
    cache, rows = make_cache(ck, B, Hkv, [2048] * (B * Hkv), [extra] * (B * Hkv), seed=3)
    return cache, rows, [m] * B, queries(m * B, Hkv * G)


def test_two_tiles_repeat_bit_for_bit(ck):
    cache, _, n_new, q = two_tiles(ck)
    a, b = run(ck, cache, n_new, q, dtype=torch.bfloat16), run(ck, cache, n_new, q, dtype=torch.bfloat16)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_two_tiles_meet_infinities_and_nan(ck):
    cache, _, n_new, q = two_tiles(ck)
    clean, clean_lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    inf, nan, n, m = float("inf"), float("nan"), 2108, n_new[0]
    finite = torch.ones_like(clean, dtype=torch.bool)
    for s, row, col, value in ((0, n - 64, 3, inf), (0, n - 40, 4, -inf), (5, n - 1, 7, nan), (77, n - 33, 127, inf), (77, n - 30, 127, -inf), (127, n - 10, 0, nan)):
        poke(cache, s, row, col, value, "v")
        b, h = divmod(s, 8)
        finite[b * m + max(0, row - (n - m)):(b + 1) * m, h * 4:h * 4 + 4, col] = False
    out, lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    assert torch.equal(lse, clean_lse) and torch.equal(torch.isfinite(out), finite) and torch.equal(out[finite], clean[finite])
    poke(cache, 9, n - 20, 3, nan, "k")
    out, lse = run(ck, cache, n_new, q, dtype=torch.bfloat16)
    at = slice(m + m - 20, 2 * m)
    assert torch.isnan(out[at, 4:8]).all() and torch.isnan(lse[at, 4:8]).all()
    lse[at, 4:8] = clean_lse[at, 4:8]
    assert torch.equal(lse, clean_lse)


def test_two_tiles_captured_over_lists_that_change(ck):
    cache, rows, n_new, q = two_tiles(ck)
    S, B = len(rows), len(n_new)
    out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=torch.bfloat16), torch.full(q.shape[:2], 3.0, device="cuda")
    chunk = ck.Chunk(n_new)
    ws = ck.chunk_attn_workspace(cache, chunk, 32)
    ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    for lens in ([2108] * S, [64 + 16 * s for s in range(S)], [100] * S, [2108 - s for s in range(S)]):
        cache.set_lengths(lens)
        g.replay()
        now = [(k[:n], v[:n]) for (k, v), n in zip(rows, lens)]
        check_rounded_once(out, lse, reference(now, q, n_new, starts(n_new), 8, D ** -0.5))
    assert ck.catekv_workspace_status(ws)["flags"] == 0


def test_two_tiles_whose_waits_run_out(ck):
    cache, rows, n_new, q = two_tiles(ck)
    out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=torch.bfloat16), torch.full(q.shape[:2], 3.0, device="cuda")
    chunk = ck.Chunk(n_new)
    ws = ck.chunk_attn_workspace(cache, chunk, 32)
    ck.catekv_test_expire_score_waits(1)
    ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    st = ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)
    assert st["flags"] == ck.STATUS_WAIT_EXPIRED and st["kernel"] == 7
    ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
    assert ck.catekv_workspace_status(ws)["flags"] == 0
    check_rounded_once(out, lse, reference(rows, q, n_new, starts(n_new), 8, D ** -0.5))


def test_doubled_rows_whose_waits_run_out(ck):
    """Few query rows over long lists: the warps also wait for one another's results."""
    cache, rows = make_cache(ck, 2, 8, [16000] * 16, [40] * 16, seed=8)
    n_new, q = [5, 3], queries(8, 32)
    out, lse = torch.full(q.shape, 3.0, device="cuda", dtype=torch.bfloat16), torch.full(q.shape[:2], 3.0, device="cuda")
    chunk = ck.Chunk(n_new)
    ws = ck.chunk_attn_workspace(cache, chunk, 32)
    for _ in range(3):
        ck.catekv_test_expire_score_waits(1)
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
        st = ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)
        assert st["flags"] == ck.STATUS_WAIT_EXPIRED and st["kernel"] == 7
        ck.catekv_chunk_attn(cache, chunk, q, out, lse, ws=ws)
        assert ck.catekv_workspace_status(ws)["flags"] == 0
        check_rounded_once(out, lse, reference(rows, q, n_new, [0, 5], 8, D ** -0.5))
