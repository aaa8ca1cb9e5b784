"""The order of experts whose keys are a few units of fp32's last place apart."""
import pytest
import torch

import paper_2608_06912_b200 as L

pytestmark = pytest.mark.gpu


def neighbours(n, low, high, gen):
    """(v, the next float above v)"""
    v = low + (high - low) * torch.rand(n, generator=gen)
    return v, torch.nextafter(v, torch.full_like(v, float("inf")))


@pytest.mark.parametrize("low,high", [(-60.0, -16.0), (-16.0, -8.0)])
@pytest.mark.parametrize("by", ["groups", "bias"])
@pytest.mark.parametrize("E", [2, 8, 64, 256])
def test_sigmoid_keys_of_neighbouring_logits(low, high, by, E):
    """Below -8 the sigmoid is e^x to 3e-4, so neighbouring logits of [-16, -8) give keys 2^-20 apart, relative to the keys, and lower
    ones more.  With an exponential of 1 unit in the last place (2^-23), a sum and a quotient (2^-24 each) two keys are at most 2^-21 off:
    the larger logit wins.  All other experts are unavailable."""
    T = 4096
    gen = torch.Generator().manual_seed(E)
    lo, hi = neighbours(T, low, high, gen)
    a, b = 0, E - 1  # in different groups; the larger one has the higher index, so a tie would show too
    x = torch.full((T, E), float("-inf"))
    x[:, a], x[:, b] = lo, hi
    p = L.route_params(k=1, score=L.ROUTE_SIGMOID, groups=2 if by == "groups" else 1, groups_kept=1)
    idx, w = torch.empty(T, 1, dtype=torch.int32, device="cuda"), torch.empty(T, 1, device="cuda")
    L.lapsum_route_forward(x.cuda(), torch.zeros(E, device="cuda") if by == "bias" else None, p, idx, w)
    wrong = (idx.cpu()[:, 0] != b).sum().item()
    assert wrong == 0, f"{wrong} of {T}"
