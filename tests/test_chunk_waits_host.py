"""CPU test of a property of the source: a warp of the chunk kernel whose wait runs out leaves as a whole.

Lanes may see a bounded wait run out, or another warp's abort flag, at different times; the code behind a wait are collectives of the whole warp
(votes, tcgen05.ld and st), which a part of a warp would wait in for good.  So no wait is taken lane by lane."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_30295_b200", "csrc", "chunk.cu")


def test_every_wait_is_the_warps():
    with open(SOURCE) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert re.findall(r"[^\n]*\bmbar_wait\([^\n]*", text) == ["  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit));"]
    assert len(re.findall(r"\bwarp_wait\(", text)) > 15
