"""The probabilities' low parts: 8-bit attention carries P as an f16 pair (22 bits) over its blocks and as three bf16 parts (24 bits) over its
tails, weighted attention as three bf16 parts.  Losing one, or pairing it with another head, has to show.

Inputs with which nearly everything else is exact.  Keys and queries have one element each, so that a logit is one product; every block's
key scale is 1; |logit| <= 1.39, 2 as a power of 2.  The value of token t is 1 at dimension t mod 128 and 0 elsewhere, so that an output
is a probability (or a sum of some).

Tolerance, in units of u = 2^-24 relative to the output, worst cases added up: the logit's scale and three multiplications on |x| <= 2, twice
for a quotient of two exponentials, 14; x + 12 - max rounded at 2^-21, times ln 2, in numerator and sum, 11; ex2.approx (2^-22) in both, 8; the
split, 4; a product's sum cut off three times by 2 u, 6; the accumulator's multiply-add, 1; two changes of maximum, 5 each; the sum of the
probabilities, 12; scale of V, reciprocal, product, 3: 69.  Bound: 72 u.  Hi and lo alone are off by up to 2^-17 (128 u) in bf16 and hi alone by
2^-12 (4096 u) in f16: the first test plants both."""
import numpy as np
import pytest
import torch

from oracle import catekv_oracle as orc
from test_gpu_q8 import _attend, _quantized, ck  # noqa: F401

U = 2.0 ** -24
BOUND = 72 * U
TYPES = [orc.Q8_E4M3, orc.Q8_INT8]
LENS = [64, 63, 128, 128 + 63, 20, 640 + 33]  # blocks alone, tails alone, both


def _case(dtype, G, lens, seed):
    """k, v: bf16 rows of every list;  q: [1, len(lens) * G, 128] bf16."""
    g = np.random.default_rng(seed)
    grid = orc.q8_grid(dtype)
    k, v = [], []
    for n in lens:
        c = g.choice(grid, n) * g.choice([-1.0, 1.0], n)
        c[::64] = grid.max()
        x, y = torch.zeros(n, 128), torch.zeros(n, 128)
        x[:, 0] = torch.from_numpy(c)
        y[torch.arange(n), torch.arange(n) % 128] = 1.0
        k.append(x.bfloat16())
        v.append(y.bfloat16())
    q = torch.zeros(1, len(lens) * G, 128)
    h = torch.arange(len(lens) * G)
    q[0, :, 0] = 1.38 / float(grid.max()) * (1 - 0.11 * (h % G)) * (1 - 2.0 * (h % 2))
    q = q.bfloat16()
    assert float(q.float().abs().max()) * grid.max() <= 1.39
    return k, v, q


def _reference(k, v, q, G, dtype=None):
    out, lse = np.zeros((len(k), G, 128)), np.zeros((len(k), G))
    weights = []
    qf = q[0].double().numpy().reshape(len(k), G, 128)
    for s in range(len(k)):
        K, V = (orc.bf16_to_f64(x[s].view(torch.int16).numpy().view(np.uint16)) if dtype is None
                else orc.q8_rows(x[s].view(torch.int16).numpy().view(np.uint16), dtype) for x in (k, v))
        for h in range(G):
            out[s, h], lse[s, h] = orc.attention(qf[s, h], K, V, 1.0)
        weights.append(orc.group_attention_weights(qf[s], K, 1.0))
    return out, lse, weights


def _close(got, want, where):
    assert np.array_equal(got[want == 0], want[want == 0]), where
    err = np.abs(got - want)[want != 0] / want[want != 0]
    assert err.max() <= BOUND, (where, err.max() / U)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_lost_part_is_beyond_the_bound(dtype):
    # planted in the oracle: outputs from probabilities that lack their last part, or have another head's
    k, v, q = _case(dtype, 4, LENS, 1)

    def parts(p, t, n):
        left, out = torch.from_numpy(p), []
        for _ in range(n):
            out.append(left.float().to(t).double())  # (p has more than 32 bits only in its first part's residual, below 2^-25 of it)
            left = left - out[-1]
        return [x.numpy() for x in out]
    for s, n in enumerate(LENS):
        x = np.stack([q[0, 4 * s + h, 0].double().item() * k[s][:, 0].double().numpy() for h in range(4)])
        p = np.exp(x - x.max(axis=1, keepdims=True))
        for t, full in ((torch.float16, 2), (torch.bfloat16, 3)):
            scaled = p * (4096.0 if t == torch.float16 else 1.0)
            part = parts(scaled, t, full)
            whole = sum(part)
            assert (np.abs(whole - scaled) / scaled).max() <= 8 * U
            lost = (np.abs(whole - part[-1] - scaled) / scaled).max()
            assert lost >= 1.2 * BOUND or n == 20, (n, t, lost / U)
            swapped = (np.abs(whole - part[1] + np.roll(part[1], 1, axis=0) - scaled) / scaled).max()
            assert swapped >= 4 * BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_eight_bit_attention(ck, dtype, G):  # noqa: F811
    k, v, q = _case(dtype, G, LENS, 2 + G)
    c = _quantized(ck, k, v, 1, len(LENS), dtype, max_new=0)
    out, lse, _ = _reference(k, v, q, G, dtype)
    for ctas in (1, 5, 40):
        o, l = _attend(ck, c, q.cuda(), ctas, sm_scale=1.0)
        o, l = o.double().cpu().numpy().reshape(out.shape), l.double().cpu().numpy().reshape(lse.shape)
        for s, n in enumerate(LENS):
            _close(o[s], out[s], (dtype, G, ctas, n))
            assert np.abs(l[s] - lse[s]).max() <= BOUND, (dtype, G, ctas, n)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_weighted_attention(ck, G):  # noqa: F811
    k, v, q = _case(orc.Q8_INT8, G, LENS, 20 + G)
    cache = ck.Cache(1, len(LENS), LENS, 0)
    for s, n in enumerate(LENS):
        o = int(cache.seg_off[s])
        cache.k_pool[o:o + n], cache.v_pool[o:o + n] = k[s].cuda(), v[s].cuda()
    cache.set_lengths(LENS)
    out, lse, weights = _reference(k, v, q, G)
    for ctas in (1, 5, 40):
        plan = ck.DecodePlan(cache, ctas)
        ck.catekv_decode_plan(cache, plan)
        w = torch.zeros(cache.total_rows, device="cuda")
        o, l = torch.empty(q.shape, device="cuda"), torch.empty(q.shape[:2], device="cuda")
        ck.catekv_decode_attn_weighted(cache, q.cuda(), plan, o, w, 1.0, ck.decode_weighted_workspace(cache, q.shape[1], plan), l, 1.0)
        o, l, w = o.double().cpu().numpy().reshape(out.shape), l.double().cpu().numpy().reshape(lse.shape), w.double().cpu().numpy()
        for s, n in enumerate(LENS):
            _close(o[s], out[s], (G, ctas, n))
            assert np.abs(l[s] - lse[s]).max() <= BOUND, (G, ctas, n)
            at = int(cache.seg_off[s])
            _close(w[at:at + n], weights[s], (G, ctas, n, "weights"))
