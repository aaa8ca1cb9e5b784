"""lapsum_sample where its integer weights are coarsest: long rows with a tail just below half a unit."""
import math

import pytest
import torch

import paper_2608_06912_b200 as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1 << 17, 1 << 18, 1 << 19, 1 << 21])
@pytest.mark.parametrize("below", [-0.02, 0.02, 0.5, 0.98, 1.02, 1.5])
def test_a_long_tail_of_weights_near_half_a_unit(vocab, below):
    """One token of weight 1 and a tail of 2^-(S + below): the sum is off by at most vocab 2^-(S + 1), S = 45 up to 2^18 tokens and one less for each doubling; the
    log probability by as much and its rounding."""
    s = min(45, 63 - int(math.log2(vocab)))
    x = torch.full((1, vocab), -(s + below) * math.log(2.0), device="cuda")
    x[0, 12345] = 0.0
    token, logprob = torch.empty(1, device="cuda", dtype=torch.int32), torch.empty(1, device="cuda")
    L.lapsum_sample(x, torch.tensor([0.05], device="cuda"), L.sample_params(), token, logprob)
    tail = math.exp(x[0, 0].double().item())
    want = -math.log1p((vocab - 1) * tail)
    assert token.item() == 12345
    assert abs(logprob.item() - want) <= vocab * 2.0 ** -(s + 1) + 2.0 ** -24 * abs(want) + 1e-12
