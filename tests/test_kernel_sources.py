"""Rules of the memory model that no run can show: read from the kernels' sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_18052_b200", "csrc")


def source(name):
    """A kernel source without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def calls(text, name):
    """The arguments of every call of a function (template arguments left out)."""
    for m in re.finditer(name + r"(?:<[^<>]*>)?\(", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        yield text[m.end():at - 1]


def test_a_vote_over_different_barriers_is_followed_by_a_warp_barrier():
    """Where the lanes of a warp wait for different barriers and vote, the vote orders no memory: a lane reads what another lane's barrier guards only
    behind __syncwarp."""
    text = source("gaf_weight_grad.cuh")
    different = [c for c in calls(text, "wg_wait_lanes") if "sh." in c]
    assert len(different) == 3 and all("lane ==" in c for c in different)
    assert not [c for c in calls(text, r"(?:wg_wait_warp|wg_wait)") if "lane" in c]
    body = text[text.index("bool wg_wait_lanes"):]
    assert re.match(r"[^}]*__all_sync\([^;]*;\s*__syncwarp\(\);\s*return", body)
