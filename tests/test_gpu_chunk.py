"""Chunks of new tokens: append and attention against the definition in 64 bits.

Tolerances.  fp32 results: a logit carries an error of about 2^-23 of its size, a probability 2^-22 (exp2; its three bf16 parts have all bits) and the
accumulators 2^-24 a step; relative L2 1e-5 leaves a factor of a few over the sum of these.  bf16 results are off by half a step of the type
more, 2^-8 of the value at most, and so is every probability on its way into the product (it is rounded to bf16 where the blocks are large): with
p (1 + e), |e| <= 2^-8, the result moves by at most 2^-8 sum p |v|.  Element by element.  lse: 1e-5 of its size."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def make_cache(ck, B, Hkv, base, extra, seed, page_order=None):
    """A cache whose lists hold base[s] + extra[s] rows, the latter in overflow pages when the capacity (base rounded up) is full; NaN everywhere
    behind the lists.  -> cache, K and V of every list as float64."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = B * Hkv
    cache = ck.Cache(B, Hkv, base, 0)
    lens = [b + e for b, e in zip(base, extra)]
    need = [max(0, -(-(n - int(c)) // 64)) for n, c in zip(lens, cache.seg_cap)]
    pages = cache.attach_pages(sum(need) + 5, max(need) + 3)
    order = np.random.default_rng(seed).permutation(sum(need) + 5)
    at = 0
    for s in range(S):
        for p in range(need[s]):
            pages.table[s, p] = order[at]
            at += 1
        pages.seg_pages[s] = need[s]
    pages.struct.next_free = sum(need) + 5
    pages.struct.released = 5
    pages.table_dev.copy_(torch.from_numpy(pages.table))
    for t in (cache.k_pool, cache.v_pool, pages.k_ovf, pages.v_ovf):
        t.fill_(float("nan"))
    cache.set_lengths(lens)
    rows = []
    for s in range(S):
        kv = []
        for pool, ovf in ((cache.k_pool, pages.k_ovf), (cache.v_pool, pages.v_ovf)):
            x = torch.randn(lens[s], D, generator=g, device="cuda").bfloat16()
            put_rows(cache, pages, pool, ovf, s, 0, x)
            kv.append(x.double())
        rows.append(kv)
    return cache, rows


def put_rows(cache, pages, pool, ovf, s, r0, x):
    cap, off = int(cache.seg_cap[s]), int(cache.seg_off[s])
    for i0 in range(0, x.shape[0]):
        r = r0 + i0
        if r < cap:
            n = min(cap - r0, x.shape[0])
            pool[off + r0:off + r0 + n] = x[:n]
            if n < x.shape[0]:
                put_rows(cache, pages, pool, ovf, s, cap, x[n:])
            return
        o = r - cap
        n = min(64 - o % 64, x.shape[0] - i0)
        pg = int(pages.table[s, o // 64])
        ovf[pg * 64 + o % 64:pg * 64 + o % 64 + n] = x[i0:i0 + n]
        if i0 + n < x.shape[0]:
            put_rows(cache, pages, pool, ovf, s, r + n, x[i0 + n:])
        return


def get_rows(cache, s, n):
    pages = cache.pages
    cap, off = int(cache.seg_cap[s]), int(cache.seg_off[s])
    out = []
    for pool, ovf in ((cache.k_pool, pages.k_ovf if pages else None), (cache.v_pool, pages.v_ovf if pages else None)):
        x = [pool[off:off + min(n, cap)]]
        for p in range(-(-max(0, n - cap) // 64)):
            pg = int(pages.table[s, p])
            x.append(ovf[pg * 64:pg * 64 + min(64, n - cap - 64 * p)])
        out.append(torch.cat(x))
    return out


def reference(rows, q, n_new, start, Hkv, scale):
    """fp64: -> out, lse with NaN where no query is, and sum p |v|."""
    T, Hq, _ = q.shape
    G = Hq // Hkv
    out = torch.full((T, Hq, D), float("nan"), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), float("nan"), dtype=torch.float64, device="cuda")
    mass = torch.zeros_like(out)
    for s, (k, v) in enumerate(rows):
        b, h = divmod(s, Hkv)
        n, m, t0 = k.shape[0], n_new[b], start[b]
        for i in range(m):
            see = n - m + i + 1
            x = q[t0 + i, h * G:(h + 1) * G].double() @ k[:see].T * scale
            z = torch.logsumexp(x, 1)
            out[t0 + i, h * G:(h + 1) * G] = torch.exp(x - z[:, None]) @ v[:see]
            mass[t0 + i, h * G:(h + 1) * G] = torch.exp(x - z[:, None]) @ v[:see].abs()
            lse[t0 + i, h * G:(h + 1) * G] = z
    return out, lse, mass


def check(got, got_lse, ref, fill):
    want, want_lse, mass = ref
    there = ~torch.isnan(want_lse)
    assert torch.equal(got[~there].float(), torch.full_like(got[~there].float(), fill))  # what belongs to no sequence is left as it was
    assert torch.equal(got_lse[~there], torch.full_like(got_lse[~there], fill))
    w, g = want[there], got[there].double()
    assert torch.isfinite(g).all()
    if got.dtype == torch.float32:
        assert float((g - w).norm() / w.norm()) <= 1e-5, float((g - w).norm() / w.norm())
    else:
        # half a step for the result and for every probability, and the fp32 error of the row beside it
        tol = (w.abs() + mass[there]) * 2.0 ** -8 + 1e-5 * w.abs().amax(dim=-1, keepdim=True) * 4
        assert ((g - w).abs() <= tol).all(), float(((g - w).abs() - tol).max())
    assert float((got_lse[there].double() - want_lse[there]).abs().max()) <= 1e-5 * max(1.0, float(want_lse[there].abs().max()))


CASES = [
    # B, Hkv, G, base, extra, n_new, layout
    (1, 1, 1, [0], [1], [1], "packed"),
    (1, 1, 4, [5], [0], [1], "packed"),
    (1, 2, 4, [128, 300], [0, 0], [4], "packed"),
    (1, 2, 8, [127, 129], [0, 0], [16], "packed"),
    (2, 1, 7, [1000, 400], [0, 0], [18, 3], "padded"),
    (1, 1, 1, [0], [200], [200], "packed"),
    (2, 2, 3, [640, 256, 0, 128], [65, 64, 1, 127], [1, 1], "packed"),
    (1, 1, 4, [4000], [0], [33], "packed"),
    (1, 1, 4, [4000], [0], [300], "packed"),
    (1, 2, 7, [384, 1024], [100, 333], [100], "packed"),
    (3, 2, 2, [128] * 6, [700] * 6, [700, 0, 1], "padded"),
    (4, 3, 5, [0, 128, 256] * 4, [90] * 12, [90, 17, 0, 52], "packed"),
    (1, 1, 6, [0], [600], [600], "packed"),
    # several tiles and several blocks for every CTA
    (2, 4, 4, [3000, 2944, 1000, 384], [0, 0, 0, 0], [300, 41], "packed"),
    (8, 8, 2, [1920], [100], [5, 1, 0, 64, 2, 3, 4, 5], "padded"),
    (5, 8, 7, [512, 0], [1500], [400, 1, 399, 2, 77], "packed"),
    (30, 8, 1, [384, 0, 128], [3], [1, 2, 3] * 10, "packed"),
]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention_of_a_chunk(ck, case, out_dtype):
    B, Hkv, G, base, extra, n_new, layout = case
    base, extra = base * (B * Hkv // len(base)), extra * (B * Hkv // len(extra))
    cache, rows = make_cache(ck, B, Hkv, base, extra, seed=len(base) + sum(n_new))
    T = max(n_new)
    start = [b * T for b in range(B)] if layout == "padded" else [sum(n_new[:b]) for b in range(B)]
    n_tokens = B * T if layout == "padded" else sum(n_new)
    chunk = ck.Chunk(n_new, start if layout == "padded" else None, n_tokens)
    g = torch.Generator(device="cuda").manual_seed(5)
    wide = torch.randn(n_tokens, Hkv * G + 3, D, generator=g, device="cuda").bfloat16()
    q = wide[:, 1:1 + Hkv * G]
    out = torch.full((n_tokens, Hkv * G, D), 3.0, device="cuda", dtype=out_dtype)
    lse = torch.full((n_tokens, Hkv * G), 3.0, device="cuda")
    ws = ck.catekv_chunk_attn(cache, chunk, q, out, lse)
    assert ck.catekv_workspace_status(ws)["flags"] == 0
    check(out, lse, reference(rows, q, n_new, start, Hkv, D ** -0.5), 3.0)
