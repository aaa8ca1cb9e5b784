"""An infinity in x reaches the weights' gradient as the formula has it: infinities of dP's sign in its own column, whatever type the gradient has."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import linear_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n,k", [(5, 24, 16), (300, 264, 136), (700, 40, 72), (20011, 11, 72), (1000, 2040, 520), (4096, 2048, 512)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("wide", [True, False])
def test_gradient_of_the_weights(rows, n, k, dtype, wide):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    inf, nan = float("inf"), float("nan")
    x = torch.randn(rows, k, device="cuda", generator=gen).to(dtype)
    w = torch.randn(n, k, device="cuda", generator=gen).to(dtype)
    x[rows // 2, 3], x[rows - 1, 7], x[0, 9] = inf, -inf, nan
    gy = torch.randn(rows, n, device="cuda", generator=gen)
    gy[gy == 0] = 1.0
    ws = L.LinearWorkspace(rows, n, k, io_dtype=L.IO_OF[dtype], out_dtype=L.IO_F32, training=True)
    gw = torch.empty(n, k, device="cuda", dtype=torch.float32 if wide else dtype)
    L.lapsum_linear_backward(gy, x, w, None, None, gw, None, ws)
    value, bound = linear_reference(x, w, None, None, "none", torch.float32, gy, gw.dtype)["grad_w"]
    assert torch.isinf(value[:, [3, 7]]).all() and torch.isnan(value[:, 9]).all()
    assert torch.equal(torch.isnan(gw), torch.isnan(value))
    assert torch.equal(gw[:, [3, 7]].double(), value[:, [3, 7]])
    rest = [c for c in range(k) if c not in (3, 7, 9)]
    assert ((gw.double() - value).abs() <= bound)[:, rest].all()
