"""Properties of the mixture-of-experts kernels that no run can show reliably, read from their sources: which loads they use for
data that the kernel before them in the stream may still be writing."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_06912_b200", "csrc")


def code(name):
    """a source file without its comments"""
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def body(text, kernel):
    """the text of one function: from its name to the brace that closes it"""
    at = text.index("{", text.index(kernel + "("))
    depth, end = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[at:end]


@pytest.mark.parametrize("name", ["routing.cuh", "experts.cuh"])
def test_no_load_promises_that_its_data_stays_constant(name):
    """The kernels are launched while the previous kernel of the stream may still write their inputs.  A load through the
    non-coherent path (ld.global.nc) promises constant data for the kernel's whole life, so the compiler may move it above
    the wait for that kernel."""
    found = re.findall(r"__ldg\(|ld\.global\.nc|io_ldg|load1\(", code(name))
    assert not found, found


def test_the_last_kernel_of_a_call_lets_no_other_start_early():
    """Its results go to any kernel of the library, some of which read their inputs through the non-coherent path: those may only
    start once it has ended."""
    text = code("experts.cuh")
    for kernel in ("experts_combine_kernel", "experts_few_down_kernel"):
        assert "launch_dependents" not in body(text, kernel), kernel
    assert "launch_dependents" not in code("routing.cuh")


def test_copies_into_a_block_s_memory_are_waited_for_though_the_block_gave_up():
    """A wait that heeds the block's give-up flag returns while the copy is on its way, and the block could end before the copy lands
    in its shared memory.  Waits for copies (of the ring on the way out, and of the epilogue's own) are bounded by time alone."""
    text = code("experts.cuh")
    assert not re.search(r"waits\.wait\(loaded\b", text)
    assert len(re.findall(r"waits\.plain\(loaded\b[^;]*, false\)", text)) == 2
    assert re.search(r"waits\.plain\(full \+ 8 \* s, phase, false\)", text)
