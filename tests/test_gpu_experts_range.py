"""fp16 experts whose gate passes the type's range: what is finite in the forward has to be finite in the backward."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import experts_reference
from tests.test_gpu_experts import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [64, 128, 256])
def test_a_gate_below_the_range_has_the_gradient_zero(rows):
    """g = -80000 or lower in three features of every expert: silu(g) and its slope are 0 there (e^-80000), so y and every gradient are
    those of the other features, within the bounds of tests/experts_util.py"""
    r = Run(150, 4, 2, 64, 72, torch.float16, training=True, seed=31, tile_rows=rows)
    r.x.copy_((r.x.float().abs() + 20).half())     # all positive, so the row of weights below gives a large sum of one sign
    r.a[:, :72] *= 1 / 32                          # the other features' gates stay of ordinary size
    for f in (0, 33, 71):
        r.a[:, f] = -64.0                          # gate: 64 inputs of 20 and more times -64: -81920 and lower
    g = r.x.float() @ r.a[0, :72].float().T
    assert g[:, 0].max() < -65520 and g[:, 1:33].abs().max() < 1000  # 65520 and more in size rounds to an fp16 infinity
    out = r()
    torch.cuda.synchronize()
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    for name, (want, bound) in ref.items():
        got = out[name].double()
        assert torch.isfinite(want).all() and torch.isfinite(got).all(), name
        assert ((got - want).abs() <= bound).all(), name
    for f in (0, 33, 71):
        assert (out["grad_w_gate_up"][:, f] == 0).all() and (out["grad_w_gate_up"][:, 72 + f] == 0).all()


def test_a_gate_above_the_range_is_an_infinity_in_the_gradient_of_up_alone():
    """g = 80000: silu(g) is kept as infinity, as a value beyond the range is everywhere, so the gradient of that up row is not finite;
    the slope is 1, and the gradients of the gate rows are right"""
    r = Run(40, 2, 1, 64, 72, torch.float16, training=True, seed=32, idx=(torch.arange(40) % 2).view(40, 1))
    r.x.copy_((r.x.float().abs() + 20).half())
    r.a[:, :72] *= 1 / 32
    r.a[:, 0] = 64.0
    r.a[:, 72] *= 2.0 ** -12                       # u small, so that h = silu(g) u stays within the range
    out = r()
    torch.cuda.synchronize()
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    want, bound = ref["y"]
    assert torch.isfinite(out["y"]).all() and ((out["y"].double() - want).abs() <= bound).all()
    want, bound = ref["grad_w_gate_up"]
    got = out["grad_w_gate_up"].double()
    assert not torch.isfinite(got[:, 72]).any()
    keep = [f for f in range(144) if f != 72]
    assert ((got - want).abs()[:, keep] <= bound[:, keep]).all()
