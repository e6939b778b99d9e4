"""Rules of the partition head's kernels that no run can show safely, read from their sources (no GPU needed)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_01000_b200", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_waits_of_the_tile_kernel_have_one_answer_for_the_whole_warp():
    # after a wait a warp goes on to instructions that all its lanes have to reach together; a lane that gave up alone
    # would leave the others waiting there
    waits = re.findall(r"\bmbar_wait\w*(?=\()", source("linear.cu"))
    assert waits.count("mbar_wait_warp") >= 5
    assert set(waits) <= {"mbar_wait_warp", "mbar_wait_quiet"}   # (the quiet one: a single lane, on its way out)
