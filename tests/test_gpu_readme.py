"""The README's decode steps run as they stand, whatever pooling the selection used."""
import os
import re

import pytest
import torch

from oracle import catekv_oracle as orc
from workloads import synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("mode,param", [(orc.POOL_NONE, 1), (orc.POOL_CHUNK, 8), (orc.POOL_SLIDING, 7)])
def test_the_steps_of_the_readme(mode, param):
    import paper_2608_30295_b200 as ck
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), flags=re.S)
    assert len(blocks) == 2
    w = synth.scaled(synth.WORKLOADS["cfg0"], n=1531, budget=200)  # chunks of 8: the last one is short
    p = synth.prefill_layer(w, 0)
    mask = p["head_mask"]
    lens = [w.budget if mask[b, h] else w.n for b in range(w.B) for h in range(w.Hkv)]
    q, kn, vn = synth.decode_inputs(w, 0, 0, "cuda", mask)
    names = {"B": w.B, "Hkv": w.Hkv, "Hq": w.Hq, "expected_lengths": lens, "q_win": p["q_win"].cuda(), "k": p["k"].cuda(), "v": p["v"].cuda(),
             "seq_len": p["seq_len"], "head_mask": mask, "budget": w.budget, "eta": w.eta, "sink": w.sink, "local": w.local, "pool_mode": mode,
             "pool_param": param, "n_tokens": 70, "k_new": kn, "v_new": vn, "q": q, "decay": 0.9,
             "out": torch.full((w.B, w.Hq, w.d), float("nan"), device="cuda")}
    exec(blocks[0], names)
    assert torch.isfinite(names["out"]).all() and names["cache"].seg_len.tolist() == names["cache"].seg_len_dev.cpu().tolist()
    names["out"].fill_(float("nan"))
    exec(blocks[1], names)
    cache, q8 = names["cache"], names["q8"]
    assert torch.isfinite(names["out"]).all()
    assert cache.seg_len.tolist() == cache.seg_len_dev.cpu().tolist() and q8.seg_len.tolist() == q8.seg_len_dev.cpu().tolist()
    assert all(n == w.budget for n, m in zip(cache.seg_len, mask.reshape(-1)) if m) and (q8.seg_len == cache.seg_len + 70).all()
    assert ck is names["ck"]
