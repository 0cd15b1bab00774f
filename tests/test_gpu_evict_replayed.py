"""A captured eviction, replayed on lists that have grown past what the captured call was given room for."""
import numpy as np
import pytest
import torch

import helpers as H
from oracle import catekv_oracle as orc
from test_gpu_evict import _weights, ck  # noqa: F401
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("long", [False, True])
def test_the_rows_kept_stay_within_their_stride(ck, in_place, long):  # noqa: F811
    """idx_out in the middle of a buffer.  In the replay lists 0 (cut to its budget), 2 (just below it) and 3 (not masked) keep more rows than
    the captured call's stride, list 1 as many: what is written is right, everything around it is as it was, and the status says so."""
    budget, sink, local = (300, 4, 32) if not long else (9300, 4, 500)
    stride = budget - 100
    lens = [stride - 50, stride - 80, stride - 60, stride]
    mask = np.array([1, 0, 1, 0], dtype=np.uint8)
    oc = H.random_cache(1, 4, lens, seed=350)
    cache = H.device_cache_from_oracle(ck, oc, 400)
    w = _weights(ck, cache, 351)
    dst = dw = None
    if not in_place:
        dst = ck.Cache(1, 4, [budget] * 4, 128)
        dw = torch.zeros(dst.total_rows, device="cuda")
    buf = torch.full((5, stride), -7, dtype=torch.int32, device="cuda")
    idx = buf.reshape(-1)[stride // 2:stride // 2 + 4 * stride].view(4, stride)
    ws = ck.evict_workspace(cache)
    ck.catekv_evict(cache, w, mask, budget, sink, local, dst, dw, None, ws)  # outside the capture first (launch attributes are set once)
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=st):
        ck.catekv_evict(cache, w, mask, budget, sink, local, dst, dw, idx, ws)
    grown = [budget + 50, stride, budget - 5, budget + 120]
    # longer lists, written as a user's own kernel would write them
    for s, n in enumerate(grown):
        assert n <= int(cache.seg_cap[s])
        o = int(cache.seg_off[s])
        for pool, name in ((cache.k_pool, "k"), (cache.v_pool, "v")):
            pool[o:o + n] = synth.randn_bf16((n, 128), "cuda", 352, name, s)
        w[o:o + n] = torch.rand(n, device="cuda")
    cache.set_lengths(grown)
    w0, k0 = w.cpu().numpy().copy(), synth.bits(cache.k_pool).copy()
    off0 = cache.seg_off.copy()
    graph.replay()
    status = ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)
    assert status["flags"] == ck.STATUS_CAPACITY and status["kernel"] == 6 and status["segment"] in (0, 2, 3)
    got = buf.cpu().numpy().reshape(-1)
    assert np.all(got[:stride // 2] == -7) and np.all(got[stride // 2 + 4 * stride:] == -7)
    out, res = idx.cpu().numpy(), dst if dst is not None else cache
    k1, w1, n1 = synth.bits(res.k_pool), (w if in_place else dw).cpu().numpy(), res.seg_len_dev.cpu().numpy()
    for s, n in enumerate(grown):
        o, t = int(off0[s]), int(res.seg_off[s])
        rows = orc.evict_indices(w0[o:o + n], sink, local, budget) if mask[s] else np.arange(n)
        assert n1[s] == len(rows)
        assert np.array_equal(out[s, :min(len(rows), stride)], rows[:stride]) and np.all(out[s, len(rows):] == -7), s
        assert np.array_equal(k1[t:t + len(rows)], k0[o:o + n][rows]) and np.array_equal(w1[t:t + len(rows)], w0[o:o + n][rows]), s
    graph.replay()  # nothing left to evict in place; into the other cache the same again
    assert ck.catekv_workspace_status(ws, clear=True, raise_on_error=False)["flags"] == ck.STATUS_CAPACITY
    assert np.array_equal(buf.cpu().numpy().reshape(-1)[:stride // 2], got[:stride // 2])
