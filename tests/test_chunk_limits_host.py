"""CPU test of chunk attention's limits: the schedule counts in 32 bits whatever a replayed call may find."""
from test_chunk_host import Fake, attend, chunk, ck  # noqa: F401 (ck: a fixture)


def test_pages_that_lists_may_be_given_later_count(ck):  # noqa: F811
    """The device's lengths decide: lists of a captured call that are given pages afterwards grow beyond what they held when it was made."""
    f = Fake(ck, [16384] * 64, pages=(1 << 20, 4))
    c = chunk(ck, [16384])  # 128 blocks of each of the 64 lists
    call = lambda: attend(ck, f, c, Hq=64, st_t=64 * 128, ws=None)
    assert call() == ck.ERR_INVALID_ARG        # 130 tiles each: within the limit, and the next check speaks
    f.pages.max_pages = 1 << 15                # 16 K tiles each: 2^27
    assert call() == ck.ERR_INVALID_ARG
    f.pages.max_pages = 1 << 20                # 512 K tiles each: 2^32
    assert call() == ck.ERR_UNSUPPORTED
    f.pages.n_pages = 1 << 15                  # there are no more pages than these
    assert call() == ck.ERR_INVALID_ARG
