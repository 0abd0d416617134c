"""What the 8-bit decode step's source has to keep to beside its results (no GPU needed)."""
import os
import re

from paper_2609_15030_gb300 import build


def loop():
    """A warp's walk over its run: from its first request to the wait for what is left after a timeout."""
    with open(os.path.join(build.CSRC, "kv8_decode.cu")) as f:
        src = f.read()
    return re.search(r"for \(int ahead = 1 - S::kStages;; \+\+ahead\) \{.*?if \(lost\) \{\n\s+// wait", src, re.S).group()


def test_lanes_are_ordered_between_a_wait_and_what_it_was_for():
    """Two lanes' asynchronous copies bring the scales that all lanes read, and one lane refills the stage that all lanes
    have read; a lane's own wait and a vote order neither, a warp barrier does."""
    wait = re.search(r"arrived<S::kStages - 2>\(\);(.*?)loader\.issue\(\);", loop(), re.S)
    assert wait is not None and "__syncwarp();" in wait.group(1)


def test_a_part_over_the_ring_waits_for_the_other_lanes():
    leave = re.search(r"arrived<0>\(\);\s+__syncwarp\(\);\s+w\.leave\(", loop())
    assert leave is not None
