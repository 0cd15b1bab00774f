"""Quantising by the device's lengths: replayed on lists that are not as the captured call saw them, and of more segments than a launch takes."""
import numpy as np
import pytest
import torch

from oracle import catekv_oracle as orc
from test_gpu_q8 import _attend, _check_attention, _check_codes, _nan_like, _oracle, _quantized, _rows, _src, ck  # noqa: F401
from workloads import synth

pytestmark = pytest.mark.gpu
TYPES = [orc.Q8_E4M3, orc.Q8_INT8]


@pytest.mark.parametrize("dtype", TYPES)
def test_a_captured_call_replays_on_lists_that_have_changed(ck, dtype):  # noqa: F811
    # captured: grid of five blocks.  Replayed: a list that ends at its capacity, one cut there past the grid, one cut there within the grid (its
    # neighbour's codes begin right behind), one that has shrunk, one that was empty
    was, grown = [70, 300, 10, 64, 0], [256, 700, 500, 5, 65]
    k, v = _rows(grown, 800)
    src = _src(ck, [torch.zeros(n, 128).bfloat16() for n in was], [torch.zeros(n, 128).bfloat16() for n in was], 1, 5, max_new=700)
    c = ck.Q8Cache(1, 5, was, 100, dtype)
    caps = [int(x) for x in c.seg_cap]
    assert caps == [256, 512, 128, 256, 128]
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    ck.catekv_q8_quantize(src, c)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        ck.catekv_q8_quantize(src, c)
    for i, n in enumerate(grown):
        o = int(src.seg_off[i])
        src.k_pool[o:o + n], src.v_pool[o:o + n] = k[i].cuda(), v[i].cuda()
    src.set_lengths(grown)
    _nan_like(c)
    graph.replay()
    there = [min(n, cap) for n, cap in zip(grown, caps)]
    assert c.seg_len_dev.cpu().tolist() == there and c.seg_len.tolist() == was
    c.seg_len[:] = there
    k, v = [x[:n] for x, n in zip(k, there)], [x[:n] for x, n in zip(v, there)]
    _check_codes(c, k, v, dtype)
    q = synth.randn_bf16((1, 10, 128), "cuda", 801, "q")
    for ctas in (1, 7):
        out, lse = _attend(ck, c, q, ctas)
        _check_attention(out, lse, _oracle(k, v, q, 1, 5, dtype), ctas)


@pytest.mark.parametrize("B,Hkv", [(16, 8), (43, 3), (256, 8), (683, 3), (600, 8)])
def test_segments_of_one_launch_and_of_several(ck, B, Hkv):  # noqa: F811
    # 128 and 129 segments, 2048 and 2049, 4800
    lens = np.random.default_rng(B).integers(0, 140, B * Hkv).tolist()
    k, v = _rows(lens, 810)
    _check_codes(_quantized(ck, k, v, B, Hkv, TYPES[B % 2], max_new=0), k, v, TYPES[B % 2])
