"""A bounded wait may run out for some lanes of a warp and not for others.  Loops that hold votes, shuffles or matrix
instructions are therefore left on an answer of the whole warp (`warp_agreed` in pipeline.cuh) and never on a lane's own: read
off the sources, since a GPU that meets the fault may hang."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_00876_b200", "csrc")


def code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def exits_on(text, what):
    """statements `if (... what ...) break;` and loop conditions that hold `what`, without an agreement of the warp"""
    found = re.findall(r"if \([^;{}]*" + what + r"[^;{}]*\) *\{?[^;{}]*;? *break;", text)
    found += re.findall(r"(?:while|for) \([^{}]*" + what + r"[^{}]*\) *\{", text)
    return [f for f in found if "warp_agreed" not in f]


def test_decode_over_4_bits_leaves_its_loops_together():
    text = code("attn_decode_kv4.cu")
    body = text[text.index("attn_decode_kv4_kernel(const K4Args a)"):text.index("attn_merge_kv4_kernel(const K4Args a)")]
    assert "arrived(" in body and "warp_agreed(!gave_up)" in body
    assert not exits_on(body, r"arrived\("), "a lane leaves on its own wait"
    # the flag is a lane's own up to the vote: between a wait and the vote nothing branches on it
    for part in body.split("arrived(")[2:]:
        until = part[:part.index("warp_agreed(!gave_up)")] if "warp_agreed(!gave_up)" in part else part
        assert not re.search(r"if \(!?gave_up\)|\(; *!gave_up", until), "a branch on a lane's own wait"


def test_packed_prompts_issue_matrix_instructions_together():
    text = code("attn_packed_tc.cu")
    issuers = text[text.index("} else if (warp == 9 || warp == 10) {"):text.index("} else if (warp < 8) {")]
    assert issuers.count("warp_agreed(ok)") >= 2 and "pk_elect()" in issuers
    assert not exits_on(issuers, r"\*abort_flag"), "a lane leaves on what it has read for itself"
    assert not re.search(r"mbar_wait_spin\((?!b, parity)", issuers), "a wait whose answer is lost"
