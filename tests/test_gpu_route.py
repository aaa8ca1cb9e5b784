"""Routing and its gradient, and the dispatch tables, against 64 bits and plain counting.

Tolerances.  A weight is a quotient of exponentials whose arguments are rounded (|l| <= 30 here: relative error below 30 x
2^-24 each, some units of 2^-24 for the exponential, the sum and the quotient): 1e-5 relative.  A gradient is w_j or s_j times
sums of k products of that accuracy: 2e-5 of the row's largest |scale gw_j|, times 1 / sum s for renormalised given scores;
a 16-bit gradient is also rounded once (half the type's epsilon).
"""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import U, chosen, dispatch_reference, route_reference

pytestmark = pytest.mark.gpu


def distinct_rows(T, E, gen, dtype):
    """Rows whose values lie on a coarse lattice in random order with some exact duplicates: no two keys are nearly equal"""
    step = 6.0 / E
    x = torch.stack([torch.randperm(E, generator=gen) for _ in range(T)]).float() * step - 3.0
    dup = torch.rand(T, E, generator=gen) < 0.05
    x = torch.where(dup, x.roll(1, 1), x)
    return x.to(dtype)


def check(x, bias, k, score="softmax", groups=1, kept=1, top=2, renorm=True, scale=1.0, seed=0, gw_dtype=torch.float32):
    T, E = x.shape
    gen = torch.Generator().manual_seed(seed)
    gw = torch.randn(T, k, generator=gen).to(gw_dtype)
    idx, w, g = route_reference(x, bias, k, score, groups, kept, top, renorm, scale, gw)
    p = L.route_params(k=k, score=L.ROUTE_SCORES[score], groups=groups, groups_kept=kept, group_top=top, renormalise=int(renorm),
                       scale=scale, io_dtype=L.IO_OF[x.dtype], grad_w_dtype=L.IO_OF[gw_dtype])
    xd = x if x.is_cuda else x.cuda()
    got_i = torch.full((T, k), 77, dtype=torch.int32, device="cuda")
    got_w, got_g = torch.full((T, k), float("nan"), device="cuda"), torch.full((T, E), float("nan"), device="cuda", dtype=x.dtype)
    L.lapsum_route_forward(xd, None if bias is None else bias.cuda(), p, got_i, got_w)
    L.lapsum_route_backward(gw.cuda(), xd, got_i, got_w, p, got_g)
    torch.cuda.synchronize()
    assert torch.equal(got_i.cpu().long(), idx)
    dw = (got_w.cpu().double() - w).abs()
    assert (dw <= 1e-5 * w.abs() + 1e-37).all(), (dw / w.abs().clamp(min=1e-30)).max()
    size = abs(scale) * gw.double().abs().max(1, keepdim=True).values
    if score == "given" and renorm:
        picked = torch.where(idx >= 0, x.cpu().double().gather(1, idx.clamp(min=0)), 0.0)
        total = picked.sum(1, keepdim=True).abs()
        size = torch.where(total > 0, size / total, size)
    bound = 2e-5 * size + U.get(x.dtype, 0.0) * g.abs() + (6e-8 if x.dtype == torch.float16 else 1e-37)  # fp16: half a subnormal
    dg = (got_g.cpu().double() - g).abs()
    assert torch.isfinite(got_g).all() and (dg <= bound).all(), (dg / bound).max()


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 3), (60, 6), (128, 8), (129, 8), (160, 6), (256, 8), (384, 10), (1000, 32), (1024, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid", "given"])
@pytest.mark.parametrize("renorm", [True, False])
def test_choice_weights_and_gradient(E, k, score, renorm):
    gen = torch.Generator().manual_seed(E + k)
    x = distinct_rows(9, E, gen, torch.float32)
    check(x + 3.5 if score == "given" else x, None, k, score, renorm=renorm, scale=2.5, seed=E)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid", "given"])
def test_storage_types_with_ties(dtype, score):
    gen = torch.Generator().manual_seed(1)
    x = (torch.randn(33, 128, generator=gen) * 2).round() / 2  # many equal logits: the lower index wins
    check((x.abs() + 0.5 if score == "given" else x).to(dtype), None, 8, score, seed=2, gw_dtype=dtype)
    check((x.abs() + 0.5 if score == "given" else x).to(dtype), None, 8, score, renorm=False, seed=2)


@pytest.mark.parametrize("groups,kept,top,E", [(2, 1, 1, 8), (4, 2, 2, 64), (8, 4, 2, 256), (8, 8, 2, 256), (32, 3, 2, 1024), (3, 2, 1, 60),
                                               (5, 2, 2, 5), (20, 7, 2, 100)])
@pytest.mark.parametrize("biased", [True, False])
def test_groups(groups, kept, top, E, biased):
    gen = torch.Generator().manual_seed(groups * E)
    x = distinct_rows(17, E, gen, torch.float32)
    bias = (torch.randperm(E, generator=gen).float() - E / 2) * (0.013 / E) if biased else None
    check(x, bias, min(kept * (E // groups), 6), "sigmoid", groups, kept, top, seed=E)


@pytest.mark.parametrize("score", ["softmax", "sigmoid", "given"])
def test_bias_enters_the_choice_only(score):
    gen = torch.Generator().manual_seed(4)
    x = distinct_rows(21, 96, gen, torch.float32)
    x = x + 3.5 if score == "given" else x
    bias = torch.randint(-3, 4, (96,), generator=gen).float() * 0.37
    check(x, bias, 5, score, seed=1)
    check(x, bias, 5, score, renorm=False, seed=1)
    bias[:90] = float("-inf")  # experts taken out of service: one choice finds no expert
    check(x[:, :], bias, 7, score, seed=1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("groups", [1, 4])
def test_experts_that_cannot_be_chosen(score, renorm, groups):
    gen = torch.Generator().manual_seed(5)
    x = distinct_rows(12, 64, gen, torch.float32)
    x[0] = float("-inf")                      # nothing left
    x[1, 1:] = float("-inf")                  # one left
    x[2, ::2] = float("-inf")
    x[3, 5:] = float("nan")                   # a NaN counts as unavailable
    x[4] = torch.finfo(torch.float32).min     # the type's lowest value is a value like any other
    x[5, :60] = torch.finfo(torch.float32).min
    x[6, 16:32] = float("-inf")               # a whole group
    check(x, None, 6, score, groups, 2 if groups > 1 else 1, 2, renorm, seed=3)


def test_extreme_logits():
    x = torch.tensor([[-200.0, -201.0, -300.0, -202.0], [500.0, 499.0, -500.0, 498.0], [0.0, -0.0, 0.0, -0.0], [1e30, -1e30, 0.0, 1e29]])
    for score in ("softmax", "sigmoid"):
        idx, w = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, 2, device="cuda")
        L.lapsum_route_forward(x.cuda(), None, L.route_params(k=2, score=L.ROUTE_SCORES[score]), idx, w)
        ri, rw, _ = route_reference(x, None, 2, score)
        assert torch.equal(idx.cpu().long(), ri)  # -0 and +0 are equal: the lower index wins
        assert ((w.cpu().double() - rw).abs() <= 1e-4 * rw + 1e-37).all(), score  # arguments of 200: 200 x 2^-24 relative, and more

    z = torch.zeros(3, 8)
    check(z, None, 3, "given", renorm=True)  # scores that sum to zero: weights and gradient 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 4, 7])
def test_strided_rows(dtype, pad):
    gen = torch.Generator().manual_seed(pad)
    wide = distinct_rows(40, 128 + pad, gen, dtype).cuda()
    check(wide[:, pad:], None, 4, "softmax")
    check(wide[:, :128], None, 4, "sigmoid", renorm=False)


def test_one_token_and_none():
    gen = torch.Generator().manual_seed(0)
    check(distinct_rows(1, 64, gen, torch.float32), None, 8)
    p = L.route_params(k=2)
    e = torch.empty(0, 8, device="cuda")
    L.lapsum_route_forward(e, None, p, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))
    L.lapsum_route_backward(torch.empty(0, 2, device="cuda"), e, torch.empty(0, 2, dtype=torch.int32, device="cuda"),
                            torch.empty(0, 2, device="cuda"), p, torch.empty(0, 8, device="cuda"))


@pytest.mark.parametrize("score", ["softmax", "sigmoid", "given"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm):
    """central differences of the 64-bit weights at a fixed choice, one logit at a time (step 1e-5: error about 1e-10)"""
    gen = torch.Generator().manual_seed(7)
    x = distinct_rows(3, 12, gen, torch.float32)
    x = x + 3.5 if score == "given" else x
    k = 4
    gw = torch.randn(3, k, generator=gen)
    p = L.route_params(k=k, score=L.ROUTE_SCORES[score], renormalise=int(renorm), scale=1.5)
    idx, w, g = torch.empty(3, k, dtype=torch.int32, device="cuda"), torch.empty(3, k, device="cuda"), torch.empty(3, 12, device="cuda")
    L.lapsum_route_forward(x.cuda(), None, p, idx, w)
    L.lapsum_route_backward(gw.cuda(), x.cuda(), idx, w, p, g)
    at = idx.cpu().long()

    def value(z):
        s = {"softmax": lambda v: torch.softmax(v, 1), "sigmoid": torch.sigmoid, "given": lambda v: v}[score](z).gather(1, at)
        return (1.5 * (s / s.sum(1, keepdim=True) if renorm else s) * gw.double()).sum()

    for t in range(3):
        for e in range(12):
            d = torch.zeros(3, 12, dtype=torch.float64)
            d[t, e] = 1e-5
            want = (value(x.double() + d) - value(x.double() - d)).item() / 2e-5
            assert abs(g[t, e].item() - want) <= 3e-5 * 1.5 * gw[t].abs().max().item(), (t, e)


def test_route_refusals():
    x = torch.zeros(4, 16, device="cuda")
    idx, w = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(4, 2, device="cuda")
    for bad in (dict(k=0), dict(k=17), dict(k=33), dict(groups=3), dict(groups=0), dict(groups=4, groups_kept=5), dict(group_top=3),
                dict(scale=0.0), dict(scale=float("nan")), dict(score=5)):
        p = L.route_params(**{"k": 2, **bad})
        n = max(1, p.k)
        with pytest.raises(L.LapsumError):
            L.lapsum_route_forward(x, None, p, torch.empty(4, p.k, dtype=torch.int32, device="cuda"), torch.empty(4, p.k, device="cuda"))
        assert n >= 1
    p = L.route_params(k=2)
    for args in ((x.half(), None, p, idx, w), (x.cpu(), None, p, idx, w), (x.t().contiguous().t(), None, p, idx, w),
                 (x, None, p, idx.long(), w), (x, torch.zeros(16, device="cuda").half(), p, idx, w)):
        with pytest.raises(TypeError):
            L.lapsum_route_forward(*args)
    for args in ((x, None, p, idx[:3], w), (x, torch.zeros(15, device="cuda"), p, idx, w)):
        with pytest.raises(ValueError):
            L.lapsum_route_forward(*args)
    with pytest.raises(L.LapsumError):
        L.lapsum_route_forward(torch.zeros(1, 1025, device="cuda"), None, p, idx[:1], w[:1])


# ------------------------------------------------------------------------------------------------------------- dispatch
def check_dispatch(idx, E, rows):
    T, k = idx.shape
    d = L.Dispatch(T, k, E, tile_rows=rows)
    d.buf.fill_(119)
    L.lapsum_dispatch(idx.cuda(), d)
    torch.cuda.synchronize()
    counts, offsets, slot_of, entry_of = dispatch_reference(idx, E, rows)
    assert d.counts.tolist() == counts and d.offsets.tolist() == offsets
    assert d.slot_of.reshape(-1).tolist() == slot_of
    got = d.entry_of.tolist()
    assert len(entry_of) <= d.capacity and got[:len(entry_of)] == entry_of and all(v == -1 for v in got[len(entry_of):])
    tiles = [e for e in range(E) for _ in range((offsets[e + 1] - offsets[e]) // rows)]
    assert d.tile_expert.tolist() == tiles + [-1] * (d.layout.tiles - len(tiles))


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 128, 8), (5, 3, 2), (33, 60, 6), (512, 128, 8), (513, 128, 8), (700, 1024, 6), (4096, 31, 1),
                                   (4097, 256, 3), (9000, 64, 8)])
@pytest.mark.parametrize("rows", [16, 32, 64, 128, 256])
def test_dispatch_tables(T, E, k, rows):
    gen = torch.Generator().manual_seed(T + E)
    check_dispatch(chosen(T, E, k, gen, drop=0.1 if T > 30 else 0.0, device="cpu"), E, rows)


def test_dispatch_with_several_chunks_per_block():
    """more than 512 chunks of 4096 entries; checked against a stable sort (integers: any difference is an error)"""
    T, k, E, rows = 700_001, 5, 37, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    idx = torch.randint(-1, E, (T, k), generator=gen, device="cuda", dtype=torch.int32)
    d = L.Dispatch(T, k, E, tile_rows=rows)
    d.buf.fill_(119)
    L.lapsum_dispatch(idx, d)
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = key.sort(dim=0, stable=True).indices
    counts = torch.bincount(key, minlength=E + 1)[:E]
    offsets = torch.cat([counts.new_zeros(1), ((counts + rows - 1) // rows * rows).cumsum(0)])
    n = int(counts.sum())
    e = key[order[:n]]
    slots = torch.arange(n, device="cuda") - (counts.cumsum(0) - counts)[e] + offsets[e]
    slot_of = torch.full_like(flat, -1)
    slot_of[order[:n]] = slots
    entry_of = torch.full((d.capacity,), -1, dtype=torch.int64, device="cuda")
    entry_of[slots] = order[:n]
    assert torch.equal(d.counts.long(), counts) and torch.equal(d.offsets.long(), offsets)
    assert torch.equal(d.slot_of.reshape(-1).long(), slot_of) and torch.equal(d.entry_of.long(), entry_of)


def test_dispatch_of_odd_batches():
    check_dispatch(torch.full((300, 4), -1, dtype=torch.int32), 8, 16)                  # nothing
    check_dispatch(torch.full((3000, 3), 7, dtype=torch.int32), 8, 64)                  # one expert takes all
    check_dispatch(torch.zeros(0, 2, dtype=torch.int32), 5, 32)                         # no token
    wild = torch.randint(-2 ** 31, 2 ** 31 - 1, (500, 2), generator=torch.Generator().manual_seed(0)).to(torch.int32)
    wild[::3] = 2
    check_dispatch(wild, 4, 16)                                                         # entries out of range are dropped


def test_dispatch_refusals():
    for T, k, E, rows in ((4, 0, 8, 16), (4, 33, 8, 16), (4, 2, 0, 16), (4, 2, 1025, 16), (4, 2, 8, 24), (-1, 2, 8, 16), (2 ** 30, 2, 8, 16)):
        with pytest.raises(L.LapsumError):
            L.lapsum_dispatch_describe(T, k, E, rows)
    d = L.Dispatch(4, 2, 8, tile_rows=16)
    with pytest.raises(ValueError):
        L.lapsum_dispatch(torch.zeros(3, 2, dtype=torch.int32, device="cuda"), d)
    with pytest.raises(TypeError):
        L.lapsum_dispatch(torch.zeros(4, 2, dtype=torch.int64, device="cuda"), d)
