"""Bulk copies of the prompt kernel of the cache end before its CTA does: a wait that gives up in any warp lets the CTA end, so the warp
that starts the copies waits for the last of them whatever its own waits have returned."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_06419_b200", "csrc")


def test_the_copying_warp_waits_for_its_last_copies():
    with open(os.path.join(CSRC, "cache_prefill.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = [m.start() for m in re.finditer(r"for \(int j = issued > LS[^;]*; j < issued; \+\+j\) drain_wait\(&bars\[LY::RAW_FULL", text)]
    assert len(at) == 1
    assert re.search(r"[;}]\s*$", text[:at[0]]), "no condition before it"
