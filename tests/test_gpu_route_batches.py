"""Routing of batches that need many blocks, in every storage type, with bias and groups, and of more than 2^31 logits.

The reference is the definition in 64 bits for all rows at once.  Tolerances: as derived in tests/test_gpu_route.py.  Where keys are computed (bias,
groups), rows in which two keys or strengths that decide differ by less than 4e-6 are drawn again: half a dozen roundings of 2^-24 on values up
to 2 each side, with room."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import U

pytestmark = pytest.mark.gpu

MARGIN = 4e-6
SCORES = {"softmax": lambda v: torch.softmax(v, 1), "sigmoid": torch.sigmoid, "given": lambda v: v}


def keys_of(x, bias, score, groups):
    """(what groups are compared by, what experts are)"""
    x = x.double()
    s = SCORES[score](x)
    s = s if bias is None else s + bias.double()
    return s, (x if bias is None else s)


def inside(s, keys, groups, kept, top):
    """the keys with those of other groups at -inf, and the gap between the last group that is kept and the next"""
    T, E = keys.shape
    strength = s.view(T, groups, -1).topk(min(top, E // groups), 2).values.sum(2)
    order = strength.sort(dim=1, descending=True, stable=True)
    gap = order.values[:, kept - 1] - order.values[:, kept] if kept < groups else torch.full((T,), 1.0, device=keys.device)
    keep = torch.zeros_like(strength, dtype=torch.bool).scatter_(1, order.indices[:, :kept], True)
    return keys.masked_fill(~keep.repeat_interleave(E // groups, 1), float("-inf")), gap


def reference(x, bias, k, score, groups, kept, top, renorm, scale, gw):
    s, keys = keys_of(x, bias, score, groups)
    if groups > 1:
        keys, _ = inside(s, keys, groups, kept, top)
    idx = keys.sort(dim=1, descending=True, stable=True).indices[:, :k]
    z = x.double().requires_grad_(True)
    w = SCORES[score](z).gather(1, idx)
    w = scale * (w / w.sum(1, keepdim=True) if renorm else w)
    (g,) = torch.autograd.grad(w, z, gw.double())
    return idx, w.detach(), g


def check(x, bias, k, score="softmax", groups=1, kept=1, top=2, renorm=True, scale=1.0, rows=slice(None), gen=None):
    """the call on all rows, the comparison on `rows`"""
    T, E = x.shape
    gw = torch.randn(T, k, device="cuda", generator=gen)
    p = L.route_params(k=k, score=L.ROUTE_SCORES[score], groups=groups, groups_kept=kept, group_top=top, renormalise=int(renorm), scale=scale,
                       io_dtype=L.IO_OF[x.dtype])
    idx, w = torch.full((T, k), 77, dtype=torch.int32, device="cuda"), torch.full((T, k), float("nan"), device="cuda")
    grad = torch.full((T, E), float("nan"), device="cuda", dtype=x.dtype)
    L.lapsum_route_forward(x, bias, p, idx, w)
    L.lapsum_route_backward(gw, x, idx, w, p, grad)
    torch.cuda.synchronize()
    x, gw, idx, w, grad = x[rows], gw[rows], idx[rows], w[rows], grad[rows]
    want_i, want_w, want_g = reference(x, bias, k, score, groups, kept, top, renorm, scale, gw)
    assert torch.equal(idx.long(), want_i)
    assert ((w.double() - want_w).abs() <= 1e-5 * want_w.abs() + 1e-37).all()
    size = abs(scale) * gw.double().abs().max(1, keepdim=True).values
    if score == "given" and renorm:
        size = size / x.double().gather(1, want_i).sum(1, keepdim=True).abs()
    bound = 2e-5 * size + U.get(x.dtype, 0.0) * want_g.abs() + (6e-8 if x.dtype == torch.float16 else 1e-37)
    assert ((grad.double() - want_g).abs() <= bound).all()


def draw(T, E, score, dtype, bias, k, groups, kept, top, gen):
    def some(n):
        x = 1.5 * torch.randn(n, E, device="cuda", generator=gen)
        return (torch.sigmoid(x) if score == "given" else x).to(dtype)

    x = some(T)
    if bias is None and groups == 1:
        return x  # compared as they stand: equal logits (16 bits have many) go to the lower index
    for _ in range(30):
        s, keys = keys_of(x, bias, score, groups)
        close = torch.zeros(T, dtype=torch.bool, device="cuda")
        if groups > 1:
            keys, gap = inside(s, keys, groups, kept, top)
            close = gap < MARGIN
        best = keys.topk(min(k + 1, E), 1).values
        step = best[:, :-1] - best[:, 1:]
        close |= ((step > 0) & (step < MARGIN)).any(1)
        if not close.any():
            return x
        x[close] = some(int(close.sum()))
    raise AssertionError("no rows with clear choices")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("given", True), ("given", False)])
@pytest.mark.parametrize("T,E,k", [(4099, 128, 8), (2050, 64, 6), (1030, 20, 3), (1500, 130, 4), (700, 256, 8), (600, 512, 10), (500, 1000, 32)])
def test_many_blocks(T, E, k, score, renorm, dtype):
    gen = torch.Generator(device="cuda").manual_seed(T)
    check(draw(T, E, score, dtype, None, k, 1, 1, 2, gen), None, k, score, renorm=renorm, scale=2.5, gen=gen)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid", "given"])
@pytest.mark.parametrize("T,E,k,groups,kept,top,biased", [(2051, 256, 8, 8, 4, 2, True), (1111, 64, 4, 4, 2, 1, True), (900, 100, 6, 20, 7, 2, True),
                                                          (300, 1024, 8, 32, 3, 2, True), (3000, 128, 8, 1, 1, 2, True), (513, 7, 2, 7, 3, 1, True),
                                                          (2051, 256, 8, 8, 4, 2, False), (1111, 64, 4, 4, 2, 1, False), (900, 100, 6, 20, 7, 2, False),
                                                          (300, 1024, 8, 32, 3, 2, False), (513, 7, 2, 7, 3, 1, False)])
def test_bias_and_groups_in_every_type(T, E, k, groups, kept, top, biased, score, dtype):
    gen = torch.Generator(device="cuda").manual_seed(E + T)
    bias = 0.05 * torch.randn(E, device="cuda", generator=gen) if biased else None
    x = draw(T, E, score, dtype, bias, min(k, E // groups * kept), groups, kept, top, gen)
    check(x, bias, min(k, E // groups * kept), score, groups, kept, top, scale=1.5, gen=gen)


@pytest.mark.parametrize("score,renorm,biased", [("softmax", True, False), ("softmax", False, False), ("sigmoid", True, True)])
def test_more_than_2_31_logits(score, renorm, biased):
    T, E, k = (1 << 21) + 77, 1024, 8
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty(T, E, device="cuda", dtype=torch.bfloat16)
    bias = 0.05 * torch.randn(E, device="cuda", generator=gen) if biased else None
    rows = torch.cat([torch.arange(300), torch.arange((1 << 21) - 300, T)]).cuda()  # offsets around 2^31 and beyond
    for part in x.split(1 << 18):
        part.normal_(generator=gen)
    x[rows] = draw(rows.numel(), E, score, torch.bfloat16, bias, k, 1, 1, 2, gen)
    assert x.numel() > 2 ** 31
    check(x, bias, k, score, renorm=renorm, rows=rows, gen=gen)
