"""Rules that no run can show: read from the kernels' sources, and from the names of what was compiled."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_18052_b200.build import LIB, build

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


def test_every_lane_polls_every_barrier_that_it_waits_for():
    """A vote orders no memory: where the lanes of a warp polled different barriers and voted, each could read only what its own one guards."""
    text = source("gaf_weight_grad.cuh")
    waits = [c for c in calls(text, "wg_wait_warp") if "sh." in c]
    assert len(waits) == 6 and not [c for c in waits if "lane" in c]
    assert not [c for c in calls(text, "wg_try") if "lane" in c or "?" in c]
    # (the one vote is that of wg_wait_warp)
    assert len(re.findall(r"__all_sync|__any_sync|__ballot_sync", text)) == 1


def test_what_passes_between_the_ctas_of_a_pair_is_ordered_at_cluster_scope():
    """Arrivals and waits without a scope order nothing beyond their CTA.  What the second CTA has in shared memory is told by a store whose completion
    releases at cluster scope; that tensor memory was read is ordered by the fences of tcgen05, at cluster scope too; the first CTA's waits acquire there."""
    text = source("gaf_weight_grad.cuh")
    assert "mbarrier.arrive.shared::cluster" not in text
    remote = re.findall(r"mbarrier\.arrive\S*shared::cluster\S*", text)
    assert remote and all(".cluster.shared::cluster" in r for r in remote)
    assert all("sh.other" in c for c in calls(text, r"(?<!void )wg_tell_first")) and "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes" in text
    assert all("sh.acc_empty" in c for c in calls(text, r"(?<!void )wg_arrive_warp_in_first"))
    crossing = re.findall(r"wg_try\S*\(&sh\.(?:other|acc_empty)", text)
    assert len(crossing) == 2 and all(c.startswith("wg_try<true>") for c in crossing)
    assert text.count("acquire.cluster") == 1 and "acquire.cluster" in text[text.index("uint32_t wg_try"):text.index("bool wg_wait_until")]


def test_every_variant_of_the_norm_is_one_that_some_width_takes():
    """The norm's kernels are compiled for the numbers of threads and tiles that by_width hands out, and for no others."""
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    build()
    names = subprocess.run([nm, "-C", LIB], capture_output=True, text=True, check=True).stdout
    short = {(32, 1), (32, 2), (32, 3), (32, 4), (128, 2), (512, 4)}
    for kernel, want in (("rms_norm_kernel", short | {(128, 4), (256, 4)}), ("rms_norm_grad_kernel", short | {(256, 2), (512, 2)})):
        found = {(int(r), int(s)) for r, s in re.findall(r"gaf::" + kernel + r"<[^>]*, (\d+), (\d+)>", names)}
        assert found == want, (kernel, found ^ want)
