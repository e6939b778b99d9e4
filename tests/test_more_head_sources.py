"""Rules of the kernels of cross entropy and experts that no run can show safely, read from their sources (no GPU needed)."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_01000_b200", "csrc")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def kernels(text):
    """{name: (signature, body)} of the kernels."""
    found = {}
    for part in re.split(r"__global__", text)[1:]:
        head, body = part[:part.index("{")], part[part.index("{"):part.find("\n}")]
        head = re.sub(r"__launch_bounds__\([^)]*\)+", "", head)
        found[re.search(r"(\w+)\s*\(", head).group(1)] = (head, body)
    return found


def early(text):
    """Kernels that are launched before the launch in front of them has ended: by name, or through a variable that holds them."""
    names = set()
    for launch in re.finditer(r"launch_early\(([^,]*),", text):
        given = launch.group(1)
        if re.fullmatch(r"\w+", given):   # what the variable was last given
            values = re.findall(r"auto %s = ([^;]*);" % given, text[:launch.start()])
            given = values[-1] if values else given
        names |= set(re.findall(r"\b((?:entropy|experts)_\w+)", given))
    return names


@pytest.mark.parametrize("name,least", [("entropy.cu", 8), ("experts.cu", 5)])
def test_kernels_that_start_early_wait_and_read_nothing_before(name, least):
    text = source(name)
    known = kernels(text)
    names = early(text) & set(known)
    # (launched by cudaLaunchKernelEx with the same attribute)
    names |= {"entropy_tiles"} & set(known)
    assert len(names) >= least, names
    for kernel in names:
        head, body = known[kernel]
        assert "ep_wait_for_launch_before()" in body, kernel
        assert "__restrict__" not in head, kernel
    assert "__ldg" not in text


def test_waits_have_one_answer_for_the_whole_warp():
    waits = re.findall(r"\bmbar_wait\w*(?=\()", source("entropy.cu"))
    assert waits.count("mbar_wait_warp") >= 10
    assert set(waits) <= {"mbar_wait_warp", "mbar_wait_quiet"}


def test_nothing_waits_on_a_flag_in_memory():
    for name in ("entropy.cu", "experts.cu"):
        assert not re.search(r"while\s*\([^)]*(volatile|atomic|ld_acquire)", source(name)), name
