"""Rules of the kernels' sources that no result can show."""

import glob
import os
import re

from paper_2607_24062_gb300 import build


def _sources():
    return {p: open(p).read() for p in sorted(glob.glob(os.path.join(build.CSRC, "*.cu*")))}


def test_aligned_cluster_barriers_follow_a_warp_sync():
    """barrier.cluster's .aligned form is undefined for a warp whose lanes come apart, and every kernel that uses it
    has blocks that one lane takes before it."""
    found = 0
    for path, text in _sources().items():
        for m in re.finditer(r"barrier\.cluster\.arrive[.a-z]*\.aligned", text):
            found += 1
            before = text[:m.start()].rstrip()
            assert re.search(r"__syncwarp\(\);\s*asm volatile\(\s*\"$", before), (path, before[-120:])
    assert found >= 1


def test_copies_of_what_others_wrote_follow_a_wait_of_every_lane():
    """Whichever lane is elected issues the copies that read other CTAs' stores to global memory. If one lane alone has waited for
    them, a vote does not order its acquire before the others' copies: every lane waits, or __syncwarp comes before the proxy
    fence."""
    found = 0
    for path, text in _sources().items():
        for m in re.finditer(r"asm volatile\(\"fence\.proxy\.async;\"", text):
            found += 1
            before = text[:m.start()]
            wait = before[before.rindex("wait_done(") - 40:]
            assert re.search(r"__all_sync\(0xffffffffu, $", wait[:40]) or re.search(r"__syncwarp\(\);\s*$", before), (path, wait)
    assert found >= 1
