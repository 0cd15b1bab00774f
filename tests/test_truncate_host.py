"""CPU test: what catekv_truncate does on the host grows with the lists, not with their square."""
import ctypes as C
import time

import numpy as np
import pytest

from test_chunk_host import Fake, ck  # noqa: F401 (ck: a fixture)


def test_a_forked_pair_does_not_slow_down_a_large_batch(ck):  # noqa: F811
    import torch
    if torch.cuda.is_available():
        pytest.skip("the call would be launched on memory that is not there")
    B, Hkv = 512, 8
    drop = np.ones(B, dtype=np.int32)

    def seconds(pair):
        f = Fake(ck, [200] * (B * Hkv), B=B, pages=(64, 4))
        if pair:  # list (1, 0) reads the first 128 rows of list (0, 0)
            f.off[Hkv], f.cap[Hkv], f.len[Hkv] = f.off[0], 128, 190
            f.give(Hkv, 0)
        best = 1.0
        for _ in range(9):
            t = time.perf_counter()
            code = ck._lib.catekv_truncate(C.byref(f.st), drop.ctypes.data, None)
            best = min(best, time.perf_counter() - t)
            assert code == ck.ERR_CUDA  # everything is decided; there is no device
        return best

    seconds(False)
    plain, forked = seconds(False), seconds(True)
    # a scan of all 4096 lists for each of them took 30 to 100 times as long as the rest of the call
    assert forked <= 4 * plain + 1e-3, (plain, forked)
