"""Gradients of fp16 layers whose upstream gradients lie anywhere in fp32's range: small as a mean over many tokens leaves them, beyond fp16's
largest number, of different size from row to row and from column to column, with an outlier."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import linear_reference

pytestmark = pytest.mark.gpu
H, F = torch.float16, torch.float32


def gradients(rows, n, k, act, gy, grad_w, grad_bias=F, want=("grad_x", "grad_w", "grad_bias"), seed=0):
    """every wanted gradient within the reference's bounds, which hold for each element from the terms of its own sum.  (dP is rounded to 11 bits, or with its
    remainder to 22; what lies 2^-40 below the largest of its row or column is less than the sums' own error.)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, k, device="cuda", generator=gen).to(H)
    w = (torch.randn(n, k, device="cuda", generator=gen) * k ** -0.5).to(H)
    b = (0.3 * torch.randn(n, device="cuda", generator=gen)).to(F)
    ws = L.LinearWorkspace(rows, n, k, activation=L.ACTIVATIONS[act], io_dtype=L.IO_F16, out_dtype=L.IO_OF[gy.dtype], training=True)
    pre, y = ws.new_pre(), torch.empty(rows, n, device="cuda", dtype=gy.dtype)
    L.lapsum_linear_forward(x, w, b, None, y, ws, pre=pre)
    got = {"grad_x": torch.full_like(x, float("nan")), "grad_w": torch.full((n, k), float("nan"), device="cuda", dtype=grad_w),
           "grad_bias": torch.full((n,), float("nan"), device="cuda", dtype=grad_bias)}
    got = {name: t if name in want else None for name, t in got.items()}
    L.lapsum_linear_backward(gy, x, w, pre, got["grad_x"], got["grad_w"], got["grad_bias"], ws)
    assert ws.status() == 0
    ref = linear_reference(x, w, b, None, act, gy.dtype, gy, grad_w, grad_bias)
    for name in want:
        value, bound = ref[name]
        t, fits = got[name], value.abs() < 0.99 * torch.finfo(got[name].dtype).max
        assert torch.isfinite(t[fits]).all(), name
        assert ((t.double() - value).abs() <= bound)[fits].all(), (name, ((t.double() - value).abs() / bound)[fits].max().item())
        beyond = value.abs() > 1.01 * torch.finfo(t.dtype).max
        assert torch.isinf(t[beyond]).all(), name
    return got


def upstream(rows, n, dtype=F, seed=1):
    return torch.randn(rows, n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("size", [1e-30, 1e-10, 1e-8, 1e-6, 1e-5, 1e-3, 1.0, 1e3, 1e6, 1e20])
@pytest.mark.parametrize("act", ["none", "silu", "relu"])
def test_upstream_gradients_of_any_size(size, act):
    gradients(700, 264, 136, act, upstream(700, 264) * size, F)


@pytest.mark.parametrize("size", [1e-8, 1e-5, 1.0])
@pytest.mark.parametrize("rows,n,k", [(1, 40, 64), (3, 1001, 264), (20011, 11, 72), (100, 9000, 64), (1000, 2040, 520), (4096, 2048, 512)])
@pytest.mark.parametrize("grad_w", [F, H])
def test_every_form_of_the_products(rows, n, k, size, grad_w):
    gradients(rows, n, k, "gelu", upstream(rows, n) * size, grad_w)


@pytest.mark.parametrize("size", [2e-7, 1e-5, 1.0])
@pytest.mark.parametrize("grad_w", [F, H])
def test_upstream_gradients_in_fp16(size, grad_w):
    gradients(900, 131, 200, "silu", upstream(900, 131).mul(size).to(H), grad_w)


@pytest.mark.parametrize("want", [("grad_x",), ("grad_w",), ("grad_bias",), ("grad_x", "grad_w"), ("grad_w", "grad_bias")])
@pytest.mark.parametrize("grad_w", [F, H])
def test_each_gradient_alone(want, grad_w):
    gradients(300, 72, 136, "gelu_tanh", upstream(300, 72) * 1e-7, grad_w, want=want)


def test_rows_and_columns_of_different_size():
    rows, n = 600, 200
    r, c = torch.arange(rows, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
    for act in ("none", "silu"):
        gradients(rows, n, 136, act, upstream(rows, n) * 10.0 ** -(r % 7).float(), F)
        gradients(rows, n, 136, act, upstream(rows, n) * 10.0 ** -(2 * (c % 9)).float(), F)


def test_an_outlier_leaves_the_other_rows_and_columns_their_digits():
    rows, n = 300, 200
    for outlier in (1e12, 1e30, float("inf"), float("nan")):
        clean, gy = upstream(rows, n) * 1e-6, upstream(rows, n) * 1e-6
        gy[37, 77] = outlier
        a, b = (gradients_of(g) for g in (clean, gy))
        others, rest = torch.arange(rows, device="cuda") != 37, torch.arange(n, device="cuda") != 77
        assert torch.equal(a[0][others], b[0][others])
        assert torch.equal(a[1][rest], b[1][rest]) and torch.equal(a[2][rest], b[2][rest])
        assert not torch.isfinite(b[0][37]).any() and (outlier < 1e38 or not torch.isfinite(b[1][77]).any())


def gradients_of(gy):
    """grad_x, grad_w and grad_bias of one layer for this upstream gradient"""
    rows, n = gy.shape
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w = (torch.randn(s, 64, device="cuda", generator=gen).to(H) for s in (rows, n))
    ws = L.LinearWorkspace(rows, n, 64, io_dtype=L.IO_F16, out_dtype=L.IO_F32, training=True)
    out = torch.empty_like(x), torch.empty(n, 64, device="cuda"), torch.empty(n, device="cuda")
    L.lapsum_linear_backward(gy, x, w, None, *out, ws)
    return out


def test_results_do_not_depend_on_scheduling():
    for grad_w in (F, H):
        a, b = (gradients(777, 515, 520, "silu", upstream(777, 515) * 1e-6, grad_w) for _ in range(2))
        assert all(torch.equal(a[name], b[name]) for name in a)


@pytest.mark.parametrize("grad_w", [F, H])
def test_a_captured_backward_finds_each_replay_s_own_sizes(grad_w):
    """what was largest in one replay, or in a call of more rows on the same workspace, has no part in the next"""
    rows, n, k = 300, 131, 72
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(rows, k, device="cuda", generator=gen).to(H)
    w = (torch.randn(n, k, device="cuda", generator=gen) * k ** -0.5).to(H)
    ws = L.LinearWorkspace(2 * rows, n, k, activation=L.ACT_SILU, io_dtype=L.IO_F16, out_dtype=L.IO_F32, training=True)
    pre, y, gy = ws.new_pre(), torch.empty(rows, n, device="cuda"), torch.empty(rows, n, device="cuda")
    L.lapsum_linear_forward(x, w, None, None, y, ws, pre=pre)
    out = torch.empty_like(x), torch.empty(n, k, device="cuda", dtype=grad_w)

    def backward(workspace, into):
        L.lapsum_linear_backward(gy, x, w, pre, into[0], into[1], None, workspace)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        backward(ws, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        backward(ws, out)
    for size in (1e8, 1.0, 1e-9, 1e3):
        gy.copy_(upstream(rows, n, seed=int(size)) * size)
        graph.replay()
        fresh = L.LinearWorkspace(rows, n, k, activation=L.ACT_SILU, io_dtype=L.IO_F16, out_dtype=L.IO_F32, training=True)
        want = torch.empty_like(out[0]), torch.empty_like(out[1])
        backward(fresh, want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), size
        big = torch.full((2 * rows, n), 1e20, device="cuda")
        x2, pre2, gx2 = x.repeat(2, 1), ws.new_pre(), torch.empty(2 * rows, k, device="cuda", dtype=H)
        pre2.zero_()
        L.lapsum_linear_backward(big, x2, w, pre2, gx2, torch.empty_like(out[1]), None, ws)
    assert ws.status() == 0
