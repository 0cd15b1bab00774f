"""Decode attention behind an append, under a plan that knows more rows than the lists hold: the appended row lies among those that the plan
would let the kernel request before the append has finished."""
import numpy as np
import pytest
import torch

import helpers as H
from oracle import catekv_oracle as orc
from test_gpu_evict import ck  # noqa: F401
from workloads import synth

pytestmark = pytest.mark.gpu


def _step(ck, oc, cache, plan, t, out, lse, G, seed):
    q, kn, vn = (synth.randn_bf16((1, h, 128), "cuda", seed, name, t) for name, h in (("q", oc.Hkv * G), ("k", oc.Hkv), ("v", oc.Hkv)))
    oc.append(synth.bits(kn), synth.bits(vn))
    torch.cuda.synchronize()
    ck.catekv_append(cache, kn, vn)
    ck.catekv_decode_attn(cache, q, plan, out, lse)
    ref, ref_lse = orc.decode_attention(oc, synth.bits(q))
    H.check_attention(out, None, lse, ref, ref_lse, t)


@pytest.mark.parametrize("ctas", [4, 40, None])
def test_lists_cut_under_their_plan(ck, ctas):  # noqa: F811
    lens, budget = [640, 300, 1000, 64], 200
    oc = H.random_cache(1, 4, lens, seed=900)
    cache = H.device_cache_from_oracle(ck, oc, 64)
    plan = ck.DecodePlan(cache, ctas or ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(cache, plan)
    w = torch.rand(cache.total_rows, device="cuda")
    wv = w.cpu().numpy()
    ck.catekv_evict(cache, w, np.ones(4, dtype=np.uint8), budget, 4, 32)
    for s, n in enumerate(lens):
        o = int(cache.seg_off[s])
        rows = orc.evict_indices(wv[o:o + n], 4, 32, budget)
        oc.k_rows[s], oc.v_rows[s] = oc.k_rows[s][rows], oc.v_rows[s][rows]
    out, lse = torch.empty(1, 12, 128, device="cuda"), torch.empty(1, 12, device="cuda")
    for t in range(60):
        _step(ck, oc, cache, plan, t, out, lse, 3, 901)


@pytest.mark.parametrize("ctas", [4, 40, None])
@pytest.mark.parametrize("sync", [False, True])
def test_a_plan_made_from_upper_bounds(ck, ctas, sync):  # noqa: F811
    lens = [121, 500, 1, 57]
    oc = H.random_cache(1, 4, lens, seed=910)
    cache = H.device_cache_from_oracle(ck, oc, 64)
    cache.seg_len += 7       # as a selection of whole chunks leaves them
    cache.struct.reserved = 1
    plan = ck.DecodePlan(cache, ctas or ck.catekv_decode_num_ctas())
    ck.catekv_decode_plan(cache, plan)
    out, lse = torch.empty(1, 12, 128, device="cuda"), torch.empty(1, 12, device="cuda")
    if sync:
        ck.catekv_cache_sync_lengths(cache)
        assert cache.seg_len.tolist() == lens
    for t in range(20):      # through the lengths that the plan was made from
        _step(ck, oc, cache, plan, t, out, lse, 3, 911)
