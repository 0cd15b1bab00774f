"""idx_out of catekv_evict as rows of a wider buffer: the library knows the distance of the rows, the binding their width."""
import numpy as np
import pytest
import torch

import helpers as H
from oracle import catekv_oracle as orc
from test_evict_host import ck  # noqa: F401


@pytest.mark.parametrize("column", [0, 40])
def test_rows_have_to_hold_what_is_kept(ck, column):  # noqa: F811
    # 64 entries are kept, a row of the view holds 60 (in the second case the last one ends with the buffer)
    cache = ck.Cache(1, 2, [100, 50], 0, "cpu")
    cache.set_lengths([100, 50])
    idx = torch.zeros(2, 100, dtype=torch.int32)[:, column:column + 60]
    with pytest.raises(ck.CatekvError) as e:
        ck.catekv_evict(cache, torch.zeros(cache.total_rows), [1, 0], 64, 0, 0, idx_out=idx, ws=torch.zeros(1 << 16, dtype=torch.uint8))
    assert e.value.code == ck.ERR_INVALID_ARG


@pytest.mark.gpu
def test_a_view_that_holds_them_is_written_and_one_in_a_capture_refused(ck):  # noqa: F811
    oc = H.random_cache(1, 3, [200, 90, 64], seed=360)
    cache = H.device_cache_from_oracle(ck, oc, 50)
    mask = np.array([1, 0, 1], dtype=np.uint8)
    w = torch.rand(cache.total_rows, device="cuda")
    w0 = w.cpu().numpy().copy()
    buf = torch.full((3, 200), -7, dtype=torch.int32, device="cuda")
    view = buf[:, 30:120]
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    ws = ck.catekv_evict(cache, w.clone(), np.zeros(3, dtype=np.uint8), 64, 4, 16)  # (keeps everything)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(ck.CatekvError) as e:
            ck.catekv_evict(cache, w, mask, 64, 4, 16, idx_out=view, ws=ws)
    assert e.value.code == ck.ERR_INVALID_ARG and cache.seg_len.tolist() == [200, 90, 64]
    ck.catekv_evict(cache, w, mask, 64, 4, 16, idx_out=view, ws=ws)
    got = buf.cpu().numpy()
    for i, n in enumerate((200, 90, 64)):
        o = int(cache.seg_off[i])
        rows = orc.evict_indices(w0[o:o + n], 4, 16, 64) if mask[i] else np.arange(n)
        assert np.array_equal(got[i, 30:30 + len(rows)], rows)
        assert np.all(got[i, :30] == -7) and np.all(got[i, 30 + len(rows):] == -7)
