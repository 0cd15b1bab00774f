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


def parity_ring(counted, uses=40, places=3, seed=0):
    """The V ring as its barriers see it, roles scheduled at random with the looking warp rarely: does that warp get through?  A wait for a use of a place
    passes when the parity of the place's completed phases says so, whichever phase that is."""
    import random
    rng = random.Random(seed)
    full, free = [0] * places, [0] * places  # completed phases; of `free`, arrivals
    need = 2 if counted else 1
    loaded = multiplied = looked = 0
    for _ in range(200 * uses):
        role = rng.choices(("load", "multiply", "look"), (8, 8, 1))[0]
        if role == "load" and loaded < uses:
            if loaded < places or free[loaded % places] >= need * (loaded // places):
                full[loaded % places] += 1
                loaded += 1
        elif role == "multiply" and multiplied < loaded:
            free[multiplied % places] += 1
            multiplied += 1
        elif role == "look" and looked < uses and full[looked % places] % 2 != (looked // places) % 2:
            if counted:
                free[looked % places] += 1
            looked += 1
    return looked == uses


def test_a_place_of_the_ring_is_free_when_the_looking_warp_has_passed_it_too():
    assert all(parity_ring(True, seed=i) for i in range(20)) and not all(parity_ring(False, seed=i) for i in range(20))
    with open(SOURCE) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert re.search(r"\(i >= kEmptyV && i < kEmptyV \+ kStagesV\) \? 2", text)  # arrivals: the products' commit, and the warp that looks
    assert len(re.findall(r"mbar_arrive\(B\(kEmptyV \+ st\)\)", text)) == 2 and len(re.findall(r"umma_commit\(B\(kEmptyV \+ st\)\)", text)) == 1


def test_the_append_of_a_chunk_does_not_signal_early():
    """Attention under a plan from before rows were taken back requests, at its start, rows that the plan knows: the append may be writing them."""
    with open(SOURCE) as f:
        text = f.read()
    body = text[text.index(" append_chunk_kernel("):text.index(" append_count_kernel(")]
    assert "pdl_wait();" in body and "pdl_launch_dependents" not in body
