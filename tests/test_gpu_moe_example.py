"""The layer of examples/moe_layer.py: soft mask, route, dispatch and experts in one chain, forward and backward."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


def load():
    spec = importlib.util.spec_from_file_location("moe_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss_and_single_tokens_agree():
    losses, apart = load().main(["--tokens", "300", "--steps", "12"])
    assert losses[-1] < 0.8 * losses[0]
    # two bf16 paths (per-slot rounding or not): a few roundings of values of size 1 apart
    assert apart <= 0.05


def test_the_chain_s_router_gradient_against_differences():
    """d loss / d logits through route and mask, against central differences in 64 bits of the same chain at the fixed choice: the mask
    by bisection, the experts' outputs as constants.  Bound: the 16-bit weights' gradient (2^-8 of the largest entry) through the
    mask's Jacobian (entries up to 1 / (2 t) = 2), twice."""
    m = load()
    T, d = 6, 64
    layer = m.MoeLayer(T, experts=8, k=2, d=d, f=64, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(T, d, device="cuda", generator=gen).to(torch.bfloat16)
    gy = torch.randn(T, d, device="cuda", generator=gen).to(torch.bfloat16)
    layer.forward(x)
    _, grad_router, _, _ = layer.backward(x, gy)
    outs = torch.zeros(T, 2, d, dtype=torch.float64, device="cuda")  # every chosen expert's output
    for t in range(T):
        for j in range(2):
            e = int(layer.idx[t, j])
            g, u = (layer.w_gate_up[e].double() @ x[t].double()).chunk(2)
            outs[t, j] = layer.w_down[e].double() @ (g * torch.sigmoid(g) * u)
    dots = (outs * gy.double()[:, None]).sum(2)

    def loss(router):
        r, temp = x.double() @ router.t(), 0.25
        lo, hi = r.min(1, keepdim=True).values - 20, r.max(1, keepdim=True).values + 20
        for _ in range(80):
            mid = (lo + hi) / 2
            v = (r - mid) / temp
            p = torch.where(v > 0, 1 - 0.5 * torch.exp(-v.abs()), 0.5 * torch.exp(-v.abs()))
            high = p.sum(1, keepdim=True) > 2
            lo, hi = torch.where(high, mid, lo), torch.where(high, hi, mid)
        w = p.gather(1, layer.idx.long())
        return ((w / w.sum(1, keepdim=True)) * dots).sum()

    direction = torch.randn(layer.router.shape, device="cuda", dtype=torch.float64, generator=gen)
    step = 1e-5
    base = layer.router.double()
    want = ((loss(base + step * direction) - loss(base - step * direction)) / (2 * step)).item()
    got = (grad_router.double() * direction).sum().item()
    reach = (x.double() @ direction.t()).abs().max().item()  # how far a logit moves along the direction
    bound = 2 * T * 2 * 2 * 2.0 ** -8 * dots.abs().max().item() * reach
    assert abs(got - want) <= bound, (got, want, bound)
