"""The sampler's variants hold what their calls can reach, read from the sources."""
import re

from tests.test_experts_source import code


def test_the_sampler_for_many_rows_holds_nothing_for_a_top_p_that_it_never_has():
    host, kernel = code("token_api.cu"), code("sample.cuh")
    assert re.search(r"many = .*!A\.top_p_row && A\.top_p >= 1;", host)
    assert "if (many) return sample_launch<T, 1024, false, false>" in host  # TOP_P
    assert "NEAR = TOP_P ? 128 : 1" in kernel and "const double p = !TOP_P ? 1.0" in kernel and "descend(TOP_P && !need_k" in kernel


def test_the_search_for_the_largest_gradient_waits_for_the_kernel_before_it():
    """and may let the next one start early, since a kernel of the same call always follows it"""
    from tests.test_experts_source import body

    text = code("linear.cuh")
    for kernel in ("linear_zero_kernel", "linear_largest_kernel"):
        assert body(text, kernel).index("pdl_wait();") < body(text, kernel).index("launch_dependents"), kernel
    host = code("linear_api.cu")
    assert re.search(r"linear_zero_kernel.*?true, grid, G, st.*?false, grid, G, st", host, re.S)
