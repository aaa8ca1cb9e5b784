"""16-bit results over contractions of several hundred thousand terms of one sign, where the tensor core's truncated additions add up.

A result has one rounding, to nearest: its relative errors are below U and as often up as down, so their mean over N results is within 6 U / sqrt(3 N) of 0 and
of what the fp32 sums leave: a round of at most 2048 terms is 128 truncated additions, each off by at most 2^-22 of a partial sum that grows evenly to the round's,
128 x 2^-22 / 2 = 2^-16 of it."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import U

pytestmark = pytest.mark.gpu


def check(got, value):
    off = (got.double() - value) / value
    u = U[got.dtype]
    assert off.abs().max() <= u + 2.0 ** -16
    assert off.mean().abs() <= 6 * u / (3 * off.numel()) ** 0.5 + 2.0 ** -16


def ones(gen, rows, cols, along, scale=1.0, dtype=torch.float16):
    """values of one sign, of another size in every column (along 0) or row, so that the results lie anywhere between two roundings"""
    size = torch.rand(*((1, cols) if along == 0 else (rows, 1)), device="cuda", generator=gen) + 1
    return torch.rand(rows, cols, device="cuda", generator=gen).mul_(0.5 * scale).add_(0.5 * scale).mul_(size).to(dtype)


def product(a, b):
    """a^T b in 64 bits, a piece at a time"""
    out = torch.zeros(a.shape[1], b.shape[1], device="cuda", dtype=torch.float64)
    for i in range(0, a.shape[0], 65536):
        out += a[i:i + 65536].double().t() @ b[i:i + 65536].double()
    return out


@pytest.mark.parametrize("rows,n,k", [(400_003, 640, 512), (65_600, 1536, 640)])
def test_gradient_of_the_weights(rows, n, k):
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, gy, w = ones(gen, rows, k, 0), ones(gen, rows, n, 0, scale=64.0 / rows), ones(gen, n, k, 0)
    ws = L.LinearWorkspace(rows, n, k, io_dtype=L.IO_F16, training=True)
    gw = torch.empty(n, k, device="cuda", dtype=torch.float16)
    L.lapsum_linear_backward(gy, x, w, None, None, gw, None, ws)
    assert ws.status() == 0
    check(gw, product(gy, x))


def test_gradient_of_the_rows():
    rows, n, k = 640, 500_000, 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, gy, w = ones(gen, rows, k, 1), ones(gen, rows, n, 1, scale=64.0 / n), ones(gen, n, k, 0)
    ws = L.LinearWorkspace(rows, n, k, io_dtype=L.IO_F16, training=True)
    gx = torch.empty(rows, k, device="cuda", dtype=torch.float16)
    L.lapsum_linear_backward(gy, x, w, None, gx, None, None, ws)
    assert ws.status() == 0
    check(gx, product(gy.t(), w))


@pytest.mark.parametrize("dtype,k", [(torch.float16, 1 << 17), (torch.bfloat16, 1 << 20)])
def test_forward(dtype, k):
    rows, n = 300, 700
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w = ones(gen, rows, k, 1, scale=64.0 / k, dtype=dtype), ones(gen, n, k, 1, dtype=dtype)
    y = torch.empty(rows, n, device="cuda", dtype=dtype)
    ws = L.LinearWorkspace(rows, n, k, io_dtype=L.IO_OF[dtype])
    L.lapsum_linear_forward(x, w, None, None, y, ws)
    assert ws.status() == 0
    check(y, product(x.t(), w.t()))
