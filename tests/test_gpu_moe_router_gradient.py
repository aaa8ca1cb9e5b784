"""The router's gradient of the layer in examples/moe_layer.py, along many directions, with a bound that follows the roundings."""
import pytest
import torch

from tests.experts_util import experts_reference
from tests.test_gpu_moe_example import load

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [3, 8])
def test_router_gradient_along_many_directions(seed):
    """d loss / d router through route and mask against central differences in 64 bits at the fixed choice, with the experts' outputs as
    constants.  Error: the weights' gradient of every choice is off by at most its bound (16-bit activations and result; independent), which
    the change of the weights along the direction carries into the sum, so sqrt(sum (bound dw)^2); the fp32 mask and its Jacobian add 1e-4
    of the terms' size.  Summed over the directions the bounds stay below a quarter of the derivatives: a gradient that is off by a
    quarter or more cannot pass along all of them."""
    m = load()
    T, E, k, d = 24, 8, 2, 64
    layer = m.MoeLayer(T, experts=E, k=k, d=d, f=64, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(T, d, device="cuda", generator=gen).to(torch.bfloat16)
    gy = torch.randn(T, d, device="cuda", generator=gen).to(torch.bfloat16)
    layer.forward(x)
    _, grad_router, _, _ = layer.backward(x, gy)
    dots, off = experts_reference(x, layer.w_gate_up, layer.w_down, layer.idx, layer.w, gy)["grad_w"]

    def weights(router):
        r, temp = x.double() @ router.t(), 0.25
        lo, hi = r.min(1, keepdim=True).values - 20, r.max(1, keepdim=True).values + 20
        for _ in range(90):
            mid = (lo + hi) / 2
            v = (r - mid) / temp
            p = torch.where(v > 0, 1 - 0.5 * torch.exp(-v.abs()), 0.5 * torch.exp(-v.abs()))
            high = p.sum(1, keepdim=True) > k
            lo, hi = torch.where(high, mid, lo), torch.where(high, hi, mid)
        w = p.gather(1, layer.idx.long())
        return w / w.sum(1, keepdim=True)

    base, step = layer.router.double(), 1e-5
    wants, bounds = [], []
    for _ in range(16):
        direction = torch.randn(base.shape, device="cuda", dtype=torch.float64, generator=gen)
        dw = (weights(base + step * direction) - weights(base - step * direction)) / (2 * step)
        want, got = (dots * dw).sum().item(), (grad_router.double() * direction).sum().item()
        bound = (off * dw).square().sum().sqrt().item() + 1e-4 * (dots * dw).abs().sum().item()
        assert abs(got - want) <= bound, (got, want, bound)
        wants.append(abs(want)), bounds.append(bound)
    assert sum(bounds) < 0.25 * sum(wants), (sum(bounds), sum(wants))
