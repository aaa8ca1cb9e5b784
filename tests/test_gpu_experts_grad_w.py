"""The routing weights' gradient in fp32, the weights' own type."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import U, experts_reference
from tests.test_gpu_experts import Run

pytestmark = pytest.mark.gpu


def both(r):
    """(16-bit, fp32) gradients of the same backward"""
    out = r()
    o = {n: torch.empty_like(out[n]) for n in ("grad_x", "grad_w_gate_up", "grad_w_down")}
    wide = torch.full_like(r.w, float("nan"))
    L.lapsum_experts_backward(r.gy, r.x, r.a, r.b, r.w, r.disp, r.saved, o["grad_x"], o["grad_w_gate_up"], o["grad_w_down"], wide, r.ws)
    torch.cuda.synchronize()
    assert r.ws.status() == 0
    for n in o:
        assert torch.equal(o[n], out[n]), n
    return out["grad_w"], wide


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,k,d,f,drop", [(1, 4, 1, 64, 64, 0.0), (300, 7, 2, 192, 320, 0.1), (70, 40, 32, 8, 8, 0.2), (1500, 8, 4, 264, 520, 0.0)])
def test_fp32_is_what_the_16_bit_gradient_is_rounded_from(dtype, T, E, k, d, f, drop):
    r = Run(T, E, k, d, f, dtype, training=True, seed=T + d, drop=drop)
    narrow, wide = both(r)
    assert torch.equal(wide.to(dtype), narrow)
    want, bound = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)["grad_w"]
    own = (U[dtype] * want.abs()).clamp(min=torch.finfo(dtype).smallest_normal * U[dtype])  # the 16-bit output's rounding: not here
    # 2^-20 of the terms' size for the fp32 sums, by Cauchy-Schwarz at most that of the roundings' bound over 6 U, times sqrt f
    slack = 2.0 ** -20 * f ** 0.5 * (bound - own) / (6 * U[dtype])
    assert ((wide.double() - want).abs() <= bound - own + slack).all()
    assert (wide[r.idx < 0] == 0).all()


def test_a_gradient_beyond_fp16():
    """<grad_y, o> is a sum over d: with a scaled loss it passes 65504 long before any other gradient does"""
    r = Run(64, 4, 2, 512, 64, torch.float16, training=True, seed=41)
    r.b.copy_(r.b.abs())                   # outputs of one sign per hidden unit, so the dot products grow with d
    r.gy.fill_(256.0)
    r.w.mul_(2.0 ** -6)                    # the other gradients carry w
    narrow, wide = both(r)
    want, bound = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)["grad_w"]
    assert want.abs().max() > 70000 and torch.isfinite(wide).all()
    assert ((wide.double() - want).abs() <= bound).all()
    assert torch.isinf(narrow[want.abs() > 70000]).all()


def test_other_types_are_refused():
    r = Run(20, 4, 2, 64, 64, training=True, seed=42)
    r()
    o = {n: torch.empty_like(r.out[n]) for n in ("grad_x", "grad_w_gate_up", "grad_w_down")}
    for bad in (r.w.half(), r.w.double()):
        with pytest.raises(TypeError):
            L.lapsum_experts_backward(r.gy, r.x, r.a, r.b, r.w, r.disp, r.saved, o["grad_x"], o["grad_w_gate_up"], o["grad_w_down"], bad, r.ws)
    with pytest.raises(ValueError):
        L.lapsum_experts_backward(r.gy, r.x, r.a, r.b, r.w, r.disp, r.saved, o["grad_x"], o["grad_w_gate_up"], o["grad_w_down"], r.w[:4], r.ws)
