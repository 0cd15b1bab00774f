"""What the page calls leave in the host's and the device's tables, and when they may be captured."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import D
from test_gpu_pages import Model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ck():
    import paper_2608_30295_b200 as pkg
    assert torch.cuda.is_available()
    return pkg.binding


def state(m):
    c, p = m.cache, m.cache.pages
    return [x.tolist() for x in (c.seg_off, c.seg_cap, c.seg_len, p.table, p.seg_pages)] + [p.struct.next_free, p.struct.released]


def test_pages_are_not_handed_out_or_moved_in_a_capture(ck):
    """The orders travel in the launch: a replay would name pages that other lists may hold by then."""
    m = Model(ck, 2, 1, [100, 100], 10, 4, 2)
    ck.catekv_pages_reserve(m.cache, 100)
    m.append([100, 100])
    m.truncate([100, 0])  # the second list's pages lie behind free ones
    before, codes = state(m), []
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for call in (lambda: ck.catekv_pages_reserve(m.cache, 100), lambda: ck.catekv_pages_compact(m.cache)):
            try:
                call()
            except ck.CatekvError as e:
                codes.append(e.code)
        ck.catekv_pages_reserve(m.cache, 10)  # there is room: nothing is handed out
    assert codes == [ck.ERR_UNSUPPORTED] * 2 and state(m) == before
    m.verify()
    assert ck.catekv_pages_compact(m.cache) == 2
    ck.catekv_pages_reserve(m.cache, 100)
    m.append([100, 100])
    m.verify()
