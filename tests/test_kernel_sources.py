"""Rules of the instruction set that no run can show to be kept: read off the kernels' sources."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1505_04956_b200", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "*.cu*")))
DRAIN = re.compile(r"commit(_pair)?\(bars \+ \w*:?:?\w*DRAIN")


@pytest.mark.parametrize("path", [p for p in FILES if DRAIN.search(open(p).read())], ids=os.path.basename)
def test_what_is_in_flight_is_committed_by_the_thread_that_issued_it(path):
    """A tcgen05.commit covers what its own thread has issued.  Where an elected lane issues the products, that lane commits before a block that gave
    up waits for them; where lane 0 does, lane 0."""
    lines = open(path).read().split("\n")
    elected = any("elect_one()" in line for line in lines)
    for i, line in enumerate(lines):
        if DRAIN.search(line):
            branch = "\n".join(lines[i - 2:i + 1])
            assert ("elect_one()" in branch) == elected and ("lane == 0" in branch) != elected, branch


def test_a_warp_whose_first_lane_alone_meets_other_blocks_synchronises_before_it_reads():
    """The meeting is an acquire by one lane; the vote that tells the others of it orders no memory, a __syncwarp() does."""
    lines = open(os.path.join(CSRC, "asgd_expert_layer.cu")).read().split("\n")
    meetings = [i for i, line in enumerate(lines) if "lane == 0" in line and "meet(a.shared" in line]
    assert meetings
    for i in meetings:
        behind = [line.split("//")[0].strip() for line in lines[i + 1:i + 4]]
        vote = next(k for k, line in enumerate(behind) if "__all_sync" in line)
        assert behind[vote + 1] == "__syncwarp();", behind
