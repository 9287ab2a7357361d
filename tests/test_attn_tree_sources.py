"""Tree attention's warps that issue matrix instructions or copies leave their loops together, and no lane waits for less than all uses
of a slot (read off the sources, since a GPU that meets the fault may hang)."""
import re

import pytest

from tests.test_wait_exits import code, exits_on


@pytest.mark.parametrize("name,issuer,softmax", [
    ("attn_tree_tc.cu", "} else if (warp >= kIssuer && warp < kIssuer + 2) {", "} else if (warp < kProducer) {"),
    ("attn_tree_rows.cu", "} else if (warp == kRwIssuer) {", "} else if (warp < 8) {")])
def test_issuers_agree_before_they_stop(name, issuer, softmax):
    text = code(name)
    part = text[text.index(issuer):text.index(softmax)]
    assert part.count("warp_agreed(ok)") >= 2
    assert not exits_on(part, r"\*abort_flag"), "a lane leaves on what it has read for itself"
    assert not re.search(r"mbar_wait_spin\((?!b, parity)", part), "a wait whose answer is lost"
    producer = text[text.index("Producer) {"):text.index(issuer)]
    assert producer.count("warp_agreed(ok)") >= 2 and not exits_on(producer, r"\*abort_flag")


def uses(order, consumers, slots):
    """For every consumer, the uses of each slot in the order it waits for them."""
    seen = {c: {} for c in consumers}
    for place, who in enumerate(order):
        for c in who:
            seen[c].setdefault(place % slots, []).append(place // slots)
    return seen


@pytest.mark.parametrize("tiles", [1, 2, 3, 7, 40])
def test_every_waiter_of_a_ring_waits_for_all_its_uses(tiles):
    """A wait by parity tells one use of a slot from the next only: who waits for a slot's uses has to wait for every one of them.
    One ring for two lanes that take alternate tiles breaks that; a ring per lane, or one that both wait through, does not."""
    together = [("A", "B")] * (2 * tiles)
    for c, slots in uses(together, "AB", 5).items():
        assert all(u == list(range(len(u))) for u in slots.values())
    own = [("A",)] * (2 * tiles)
    assert all(u == list(range(len(u))) for u in uses(own, "A", 3)["A"].values())
    if tiles >= 7:
        apart = [("AB"[(k + 1) // 2 % 2],) for k in range(2 * tiles)]
        assert any(u != list(range(len(u))) for s in uses(apart, "AB", 5).values() for u in s.values())
