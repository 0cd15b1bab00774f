"""8-bit attention: one CTA works through many lists, and each list's result is that of the list alone, bit for bit.

A list that is not cut is shared out over the warps of its CTA in the same way wherever it lies, so nothing of its neighbours may show: not
where a warp has no unit in one of them, and not where the lists are empty."""
import numpy as np
import pytest
import torch

from oracle import catekv_oracle as orc
from test_gpu_q8 import _attend, _check_attention, _oracle, _quantized, _rows, ck  # noqa: F401
from workloads import synth

pytestmark = pytest.mark.gpu


def _uncut(plan, n_segs):
    buf = plan.host.numpy()
    off_seg = int(buf[:48].view(np.int32)[10])
    return buf[off_seg:off_seg + 16 * n_segs].view(np.int32).reshape(n_segs, 4)[:, 1] <= 1


@pytest.mark.parametrize("dtype", [orc.Q8_E4M3, orc.Q8_INT8])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_every_list_is_as_it_is_alone(ck, dtype, G):  # noqa: F811
    B, Hkv = 20, 8
    rng = np.random.default_rng(700 + G)
    lens = rng.integers(0, 101, B * Hkv)
    lens[::7] = rng.integers(150, 400, len(lens[::7]))                 # a list that keeps every warp busy,
    lens[1::7] = 0                                                     # one that leaves them all idle,
    lens[2::7] = rng.integers(0, 2, len(lens[2::7]))                   # and one for the first at most
    k, v = _rows(lens.tolist(), 701)
    c = _quantized(ck, k, v, B, Hkv, dtype, max_new=0)
    q = synth.randn_bf16((B, Hkv * G, 128), "cuda", 702, "q", G)
    want, wlse = torch.zeros(B * Hkv, G, 128, device="cuda"), torch.full((B * Hkv, G), float("-inf"), device="cuda")
    for s, n in enumerate(lens):
        if n:
            alone = _quantized(ck, [k[s]], [v[s]], 1, 1, dtype, max_new=0)
            o, l = _attend(ck, alone, q.reshape(B * Hkv, G, 128)[s][None].contiguous(), 1)
            want[s], wlse[s] = o[0], l[0]
    _check_attention(want.reshape(q.shape), wlse.reshape(q.shape[:2]), _oracle(k, v, q, B, Hkv, dtype))
    for ctas in (1, 2, 5):
        plan = ck.DecodePlan(c, ctas)
        ck.catekv_q8_decode_plan(c, plan)
        at = torch.from_numpy(_uncut(plan, B * Hkv)).cuda()
        assert int((~at).sum()) < ctas
        for i in range(40):
            o, l = _attend(ck, c, q, plan=plan)
            assert torch.equal(o.reshape(want.shape)[at], want[at]), (ctas, i)
            assert torch.equal(l.reshape(wlse.shape)[at], wlse[at]), (ctas, i)
