"""lapsum_linear_forward / lapsum_linear_backward against 64 bits: every tile form, rows from one on, ragged widths, strides, types."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import linear_reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def strided(rows, cols, dtype, extra, gen, scale=1.0):
    """a rows x cols view of rows cols + extra apart; the memory between the rows is NaN"""
    buf = torch.full((rows, cols + extra), float("nan"), device="cuda", dtype=dtype)
    buf[:, :cols] = (scale * torch.randn(rows, cols, device="cuda", generator=gen)).to(dtype)
    return buf[:, :cols]


def run(rows, n, k, dtype="bf16", act="none", bias=None, residual=False, out="same", backward=False, grad_w="same", extra=0, seed=0, ws_rows=None,
        in_place=False, pre_dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    odt = dt if out == "same" else DT[out]
    x = strided(rows, k, dt, 8 * extra, gen)
    w = (torch.randn(n, k, device="cuda", generator=gen) * k ** -0.5).to(dt)
    b = None if bias is None else (0.3 * torch.randn(n, device="cuda", generator=gen)).to(dt if bias == "same" else DT[bias])
    res = strided(rows, n, odt, 3 * extra, gen) if residual else None
    y = strided(rows, n, odt, 5 * extra, gen)
    r_in = res.clone() if residual else None
    if in_place:
        y = res
    ws = L.LinearWorkspace(ws_rows or rows, n, k, activation=L.ACTIVATIONS[act], io_dtype=L.IO_OF[dt], out_dtype=L.IO_OF[odt], training=backward,
                           pre_dtype=L.IO_OF[pre_dtype])
    pre = ws.new_pre() if backward else None
    y_base = y._base if y._base is not None else y
    gap = y_base[:, n:].clone()
    L.lapsum_linear_forward(x, w, b, res, y, ws, pre=pre)
    got = {"y": y}
    gy = None
    if backward:
        gy = strided(rows, n, odt, 7 * extra, gen)
        gwt = dt if grad_w == "same" else DT[grad_w]
        got["grad_x"], got["grad_w"] = strided(rows, k, dt, extra, gen), torch.full((n, k), float("nan"), device="cuda", dtype=gwt)
        if b is not None:
            got["grad_bias"] = torch.full_like(b, float("nan"))
        L.lapsum_linear_backward(gy, x, w, pre, got["grad_x"], got["grad_w"], got.get("grad_bias"), ws)
    assert ws.status() == 0
    assert torch.equal(torch.isnan(y_base[:, n:]), torch.isnan(gap))  # what lies between the rows stays as it was
    ref = linear_reference(x, w, b, r_in, act, odt, gy, got["grad_w"].dtype if backward else None, b.dtype if b is not None else None, pre_dtype)
    for name, t in got.items():
        value, bound = ref[name]
        err = (t.double() - value).abs()
        assert torch.isfinite(t).all(), name
        worst = (err / bound).max().item()
        assert worst <= 1, (name, worst, err.max().item())
    return got


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 16, 17, 48, 65, 129, 300, 1021])
@pytest.mark.parametrize("n,k", [(1, 8), (7, 72), (129, 200), (1003, 520)])
def test_forward_of_every_number_of_rows(rows, n, k):
    run(rows, n, k, bias="same", residual=True, extra=1, seed=rows)


@pytest.mark.parametrize("rows,n,k", [(48, 40000, 256), (300, 5000, 2048), (2048, 2048, 512), (4096, 128, 1024), (1000, 4104, 264), (16, 2048, 4096)])
@pytest.mark.parametrize("dtype,out", [("bf16", "same"), ("f16", "f32")])
def test_forward_of_large_shapes(rows, n, k, dtype, out):
    run(rows, n, k, dtype=dtype, out=out, bias="f32", seed=n)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype,out,bias,grad_w", [("bf16", "same", "same", "f32"), ("f16", "f32", "f32", "same")])
@pytest.mark.parametrize("rows,n,k", [(1, 40, 64), (3, 1001, 264), (130, 72, 136), (777, 515, 520)])
def test_forward_and_backward(rows, n, k, dtype, out, bias, grad_w, act):
    run(rows, n, k, dtype=dtype, act=act, bias=bias, residual=True, out=out, backward=True, grad_w=grad_w, seed=rows + n)


@pytest.mark.parametrize("rows,n,k", [(1, 1, 8), (5, 3, 8), (64, 8, 64), (65, 64, 128), (2000, 24, 72), (9, 2056, 1032)])
def test_backward_of_small_and_strided_shapes(rows, n, k):
    run(rows, n, k, act="silu", bias="same", backward=True, extra=1, seed=n)
    run(rows, n, k, act="none", backward=True, extra=0, seed=n)


@pytest.mark.parametrize("rows,n,k", [(4096, 2048, 1024), (3000, 1024, 2048), (8192, 512, 512)])
def test_backward_of_large_shapes(rows, n, k):
    run(rows, n, k, act="gelu", bias="f32", residual=True, backward=True, grad_w="f32", seed=n)


def test_fewer_rows_than_the_workspace_and_the_residual_in_place():
    run(100, 264, 136, ws_rows=512, residual=True, in_place=True)
    run(3, 264, 136, ws_rows=512, act="silu", bias="same", backward=True)
    run(70, 264, 136, ws_rows=512, act="silu", bias="same", backward=True)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_a_pre_activation_kept_in_16_bits(act):
    run(200, 515, 136, act=act, bias="same", backward=True, grad_w="f32", pre_dtype=torch.bfloat16)
    run(3, 40, 136, act=act, bias="f32", backward=True, pre_dtype=torch.bfloat16)


@pytest.mark.parametrize("rows,n,k", [(1000, 136, 16384), (20000, 264, 256)])
def test_fp32_results_keep_fp32_digits_over_a_long_contraction(rows, n, k):
    """in the 2-norm: the rounds of 512 keep the truncated additions' error below 32 x 2^-25, with dW's rounding remainder 2^-18"""
    got = run(rows, n, k, act="silu", bias="f32", out="f32", backward=True, grad_w="f32")
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = strided(rows, k, torch.bfloat16, 0, gen)
    w = (torch.randn(n, k, device="cuda", generator=gen) * k ** -0.5).bfloat16()
    b = 0.3 * torch.randn(n, device="cuda", generator=gen)
    strided(rows, n, torch.float32, 0, gen)
    ref = linear_reference(x, w, b, None, "silu", torch.float32, strided(rows, n, torch.float32, 0, gen))
    for name in ("y", "grad_w", "grad_bias"):
        value = ref[name][0]
        assert (got[name].double() - value).norm() <= 2.0 ** -17 * value.norm(), name


@pytest.mark.parametrize("rows,n,k,out", [(1021, 2048, 5632, "same"), (1000, 2040, 4104, "f32"), (129, 300, 2048, "f32"), (512, 1024, 1000, "same"), (300, 4000, 8192, "same")])
def test_shared_contractions(rows, n, k, out):
    run(rows, n, k, bias="same", residual=True, out=out, extra=1, seed=k)
    run(rows, n, k, act="silu", bias="f32", out=out, backward=True, grad_w="f32", seed=k)


@pytest.mark.parametrize("rows,n,k,grad_w,act", [(20011, 11, 72, "f32", "none"), (9000, 130, 256, "same", "silu"), (300, 6011, 136, "f32", "gelu"), (40, 9000, 64, "same", "none"),
                                                   (16384, 1, 8, "f32", "silu"), (3000, 64, 520, "same", "relu")])
def test_gradients_of_few_tiles_and_a_long_contraction(rows, n, k, grad_w, act):
    a = run(rows, n, k, act=act, bias="f32", backward=True, grad_w=grad_w, extra=1, seed=n)
    b = run(rows, n, k, act=act, bias="f32", backward=True, grad_w=grad_w, extra=1, seed=n)
    assert all(torch.equal(a[name], b[name]) for name in a)


def test_no_rows():
    ws = L.LinearWorkspace(4, 16, 8, training=True)
    e = torch.empty(0, 8, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(0, 16, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(16, 8, device="cuda").bfloat16()
    L.lapsum_linear_forward(e, w, None, None, y, ws)
    gw, gb = torch.full((16, 8), 7.0, device="cuda"), torch.full((16,), 7.0, device="cuda", dtype=torch.bfloat16)
    L.lapsum_linear_backward(y, e, w, None, e, gw, gb, ws)
    assert not gw.any() and not gb.any()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gradients_against_differences(act):
    """the loss <gy, y> in fp32 outputs, along single weights and biases.  A step h of 2^-4 keeps the inputs exact; the quotient is off by
    h^2 |third derivative| / 6 <= 2^-8 * 2 / 6 * |gy x^3| and the gradient by the bounds of the formula's test."""
    rows, n, k = 6, 16, 16
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = (torch.randint(-8, 9, (rows, k), device="cuda", generator=gen) / 8).bfloat16()
    w = (torch.randint(-8, 9, (n, k), device="cuda", generator=gen) / 16).bfloat16()
    b = (torch.randint(-8, 9, (n,), device="cuda", generator=gen) / 8).float()
    gy = torch.randn(rows, n, device="cuda", generator=gen)
    ws = L.LinearWorkspace(rows, n, k, activation=L.ACTIVATIONS[act], out_dtype=L.IO_F32, training=True)
    pre, y = ws.new_pre(), torch.empty(rows, n, device="cuda")

    def loss(w_, b_):
        L.lapsum_linear_forward(x, w_, b_, None, y, ws, pre=pre)
        return (gy.double() * y.double()).sum().item()

    loss(w, b)
    gw, gb = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    L.lapsum_linear_backward(gy, x, w, pre, None, gw, gb, ws)
    h = 2.0 ** -4
    p = x.double() @ w.double().t() + b.double()
    for i in range(8):
        if act == "relu" and p[:, i].abs().min() < 2 * h:
            continue  # a step would cross the kink
        up, down = b.clone(), b.clone()
        up[i] += h
        down[i] -= h
        quotient = (loss(w, up) - loss(w, down)) / (2 * h)
        room = (gy[:, i].abs().double() * (2.0 ** -8 / 3 + 1.2 * 2.0 ** -8 * p[:, i].abs() + 2.0 ** -8)).sum().item() + 1e-4
        assert abs(quotient - gb[i].item()) <= room, (act, i)
        up, down = w.clone(), w.clone()
        up[i, 3] += h
        down[i, 3] -= h
        assert (up[i, 3] - down[i, 3]).item() == 2 * h
        quotient = (loss(up, b) - loss(down, b)) / (2 * h)
        assert abs(quotient - gw[i, 3].item()) <= room, (act, i)


@pytest.mark.parametrize("rows,n,k", [(48, 1000, 512), (16, 64, 4096), (600, 600, 600), (2048, 2048, 256)])
def test_results_do_not_depend_on_scheduling(rows, n, k):
    a = run(rows, n, k, act="silu", bias="same", residual=True, backward=True)
    b = run(rows, n, k, act="silu", bias="same", residual=True, backward=True)
    assert all(torch.equal(a[name], b[name]) for name in a)


def test_infinite_and_nan_inputs_reach_their_own_rows_alone():
    rows, n, k = 40, 72, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, k, device="cuda", generator=gen).half()
    w = (torch.randn(n, k, device="cuda", generator=gen) / 8).half()
    ws = L.LinearWorkspace(rows, n, k, activation=L.ACT_GELU_TANH, io_dtype=L.IO_F16, training=True, pre_dtype=L.IO_F16)
    clean, y = torch.empty(rows, n, device="cuda", dtype=torch.float16), torch.empty(rows, n, device="cuda", dtype=torch.float16)
    pre = ws.new_pre()
    L.lapsum_linear_forward(x, w, None, None, clean, ws, pre=pre)
    bad = x.clone()
    bad[3, 5], bad[7, 0] = float("nan"), 60000.0
    bad[7, 1:] = 0
    L.lapsum_linear_forward(bad, w * 64, None, None, y, ws, pre=pre)
    assert torch.isnan(y[3]).all()
    gy, gx = torch.ones_like(y), torch.empty_like(x)
    L.lapsum_linear_backward(gy, bad, w, pre, gx, None, None, ws)
    assert torch.isinf(pre[7]).any() and torch.isfinite(gx[7]).all()  # a pre-activation beyond the type's range has the slope's limit
    assert torch.isnan(gx[3]).all() and torch.isfinite(gx[[i for i in range(rows) if i != 3]]).all()
    L.lapsum_linear_forward(bad, w, None, None, y, ws, pre=pre)
    others = [i for i in range(rows) if i not in (3, 7)]
    assert torch.equal(y[others], clean[others])
