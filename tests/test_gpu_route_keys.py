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


@pytest.mark.parametrize("by", ["logits", "bias", "groups"])
def test_an_infinite_logit_under_softmax(by):
    """its weights are NaN; where the scores themselves are the keys, a NaN key is never chosen.  Other rows do not notice."""
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(5, 16, generator=gen).cuda()
    clean = x.clone()
    x[2, 3] = float("inf")
    bias = torch.zeros(16, device="cuda") if by == "bias" else None
    p = L.route_params(k=4, groups=4 if by == "groups" else 1, groups_kept=2 if by == "groups" else 1)
    got = []
    for v in (x, clean):
        idx, w = torch.empty(5, 4, dtype=torch.int32, device="cuda"), torch.empty(5, 4, device="cuda")
        L.lapsum_route_forward(v, bias, p, idx, w)
        got.append((idx.cpu(), w.cpu()))
    others = [0, 1, 3, 4]
    assert torch.equal(got[0][0][others], got[1][0][others]) and torch.equal(got[0][1][others], got[1][1][others])
    if by == "logits":
        assert got[0][0][2, 0] == 3 and torch.isnan(got[0][1][2]).all()
    else:
        assert (got[0][0][2] == -1).all() and (got[0][1][2] == 0).all()
