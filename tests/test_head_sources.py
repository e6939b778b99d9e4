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


def test_kernels_that_start_early_read_nothing_that_may_be_read_before_their_wait():
    # what the launch before writes is there only after the wait; a load through __restrict__ or __ldg promises the compiler
    # that nothing writes there, so that it may move the load ahead of the wait
    kernels = 0
    for name in ("norm.cu", "route.cu", "linear.cu"):
        for kernel in re.split(r"__global__", source(name))[1:]:
            body = kernel[:kernel.find("\n}")]
            if "ep_wait_for_launch_before()" not in body:
                continue
            kernels += 1
            assert "__restrict__" not in body[:body.index("{")], (name, body[:120])
    assert kernels == 4
    assert "__ldg" not in source("linear.cu") and "__ldg" not in source("rows.cuh")
