"""The sampler's variants hold what their calls can reach, read from the sources."""
import re

from tests.test_experts_source import code


def test_the_sampler_for_many_rows_holds_nothing_for_a_top_p_that_it_never_has():
    host, kernel = code("token_api.cu"), code("sample.cuh")
    assert re.search(r"many = .*!A\.top_p_row && A\.top_p >= 1;", host)
    assert "if (many) return sample_launch<T, 1024, false, false>" in host  # TOP_P
    assert "NEAR = TOP_P ? 128 : 1" in kernel and "const double p = !TOP_P ? 1.0" in kernel and "descend(TOP_P && !need_k" in kernel
