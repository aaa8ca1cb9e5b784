"""gelu and its slope keep their digits where they are tiny: far to the left the value is 0.5 x erfc(-x / sqrt 2), never a difference of two near ones.

The argument of erfc is off by 2^-23 of itself (the constant and the product), which its condition, below x^2 + 2, carries on; erfc has 4 ulp, the products
another: (x^2 + 8) 2^-23 of the value.  The slope is the difference of x phi(x), whose exponential is as exact, and Phi(x): from x = -1 on their sizes
add up to at most 5 times the slope."""
import math

import pytest
import torch

import paper_2608_06912_b200 as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 4, 48])
def test_gelu_far_to_the_left(rows):
    p = -torch.linspace(1.0, 12.5, 93, dtype=torch.float64).bfloat16().double()
    n, k = len(p), 8
    x, w = torch.zeros(rows, k, device="cuda").bfloat16(), torch.zeros(n, k, device="cuda").bfloat16()
    x[:, 0], w[:, 0] = 1.0, p.cuda().bfloat16()  # P is p itself
    ws = L.LinearWorkspace(rows, n, k, activation=L.ACT_GELU, out_dtype=L.IO_F32, training=True)
    y, pre = torch.empty(rows, n, device="cuda"), ws.new_pre()
    L.lapsum_linear_forward(x, w, None, None, y, ws, pre=pre)
    gy, gb = torch.zeros(rows, n, device="cuda"), torch.empty(n, device="cuda")
    gy[0] = 1.0
    L.lapsum_linear_backward(gy, x, w, pre, None, None, gb, ws)
    phi = torch.tensor([math.exp(-0.5 * v * v) / math.sqrt(2 * math.pi) for v in p.tolist()], dtype=torch.float64)
    below = torch.tensor([0.5 * math.erfc(-v * math.sqrt(0.5)) for v in p.tolist()], dtype=torch.float64)
    room = (p * p + 8) * 2.0 ** -23
    off = ((y.double().cpu() - p * below) / (p * below)).abs()
    assert (off <= room).all(), (off / room).max()
    slope = below + p * phi
    off = ((gb.double().cpu() - slope) / slope).abs()
    assert (off <= 5 * room).all(), (off / room).max()
