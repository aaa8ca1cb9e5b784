"""Properties of the dense operators' kernels that no run can show reliably, read from their sources."""
import re

import pytest

from tests.test_experts_source import body, code


@pytest.mark.parametrize("name", ["linear.cuh", "sample.cuh", "embed.cuh", "tensor_core.cuh"])
def test_no_load_promises_that_its_data_stays_constant(name):
    """The kernels start while the previous kernel of the stream may still write their inputs."""
    found = re.findall(r"__ldg\(|ld\.global\.nc|io_ldg|load1\(", code(name))
    assert not found, found


def test_the_last_kernel_of_a_call_lets_no_other_start_early():
    """Its results go to any kernel of the library, some of which read their inputs through the non-coherent path."""
    text = code("linear.cuh")
    for kernel in ("linear_kernel", "linear_few_kernel", "linear_bias_kernel", "linear_parts_kernel"):
        assert "launch_dependents" not in body(text, kernel), kernel
    text = code("embed.cuh")
    for kernel in ("embed_forward_kernel", "embed_join_kernel"):
        assert "launch_dependents" not in body(text, kernel), kernel
    assert "if (P.tokens > EMBED_LONG) asm volatile(\"griddepcontrol.launch_dependents" in body(text, "embed_grad_kernel")
    assert "launch_dependents" not in code("sample.cuh")


def test_every_kernel_waits_for_the_one_before_it():
    for name, kernels in (("linear.cuh", ("linear_kernel", "linear_few_kernel", "linear_grad_kernel", "linear_bias_kernel", "linear_parts_kernel")),
                          ("embed.cuh", ("embed_forward_kernel", "embed_sort_kernel", "embed_grad_kernel", "embed_join_kernel")),
                          ("sample.cuh", ("sample_kernel",))):
        for kernel in kernels:
            assert "pdl_wait();" in body(code(name), kernel), kernel


def test_copies_into_a_block_s_memory_are_waited_for_though_the_block_gave_up():
    assert re.search(r"waits\.plain\(full \+ 8 \* s, phase, false\)", body(code("linear.cuh"), "linear_kernel"))


def test_no_wait_of_the_sampler_is_a_loop():
    """blocks of a row wait for one another at cluster barriers alone, and each arrives at as many as the others: no flag is polled"""
    assert not re.search(r"while\s*\(\s*(!|ld|far|\*)", code("sample.cuh"))
