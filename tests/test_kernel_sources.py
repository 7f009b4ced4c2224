"""Rules that the kernels' sources keep and no run can show: what would break them faults or hangs a GPU."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_12528_b200", "csrc")


def code(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


ELECTING = [os.path.basename(p) for p in sorted(glob.glob(os.path.join(CSRC, "*.cu"))) if "elect.sync" in code(p)]


@pytest.mark.parametrize("name", ELECTING)
def test_warps_that_elect_a_lane_leave_their_waits_together(name):
    # elect.sync names all 32 lanes: a warp of which some lanes have left a wait that ran out must not come to it.
    # So there is one place that polls a barrier, and its answer is the warp's.
    text = code(os.path.join(CSRC, name))
    assert len(re.findall(r"\bmbar_try_wait\(", text)) == 1
    wait = re.search(r"auto wait = \[&\]\(uint64_t\* bar, uint32_t parity\) -> bool \{(.*?)\n    \};", text, re.S)
    assert "mbar_try_wait(bar, parity)" in wait.group(1)
    assert re.findall(r"return [^;]*;", wait.group(1)) == ["return __all_sync(0xFFFFFFFFu, there);"]


def test_some_kernel_elects():
    assert ELECTING == ["prefix.cu"]
