"""lapsum_embed_forward / lapsum_embed_backward: values bit for bit, gradients against 64 bits."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import embed_reference

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def forward(ids, table, scale, out=None):
    out = torch.full((ids.shape[0], table.shape[1]), float("nan"), device="cuda", dtype=table.dtype) if out is None else out
    L.lapsum_embed_forward(ids, table, out, scale=scale)
    real = (ids >= 0) & (ids < table.shape[0])
    want = (table.float()[torch.where(real, ids, 0).long()] * scale).to(table.dtype)
    want[~real] = 0
    assert torch.equal(out, want)


def backward(ids, vocab, d, dtype, scale=1.0, skip=-1, wide=False, ws=None, stride=None, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, dt = ids.shape[0], DT[dtype]
    g = torch.randn(n, stride or d, device="cuda", generator=gen).to(dt)[:, :d]
    grad = torch.full((vocab, d), float("nan"), device="cuda", dtype=torch.float32 if wide else dt)
    ws = ws or L.EmbedWorkspace(n, vocab, d)
    L.lapsum_embed_backward(g, ids, grad, ws, scale=scale, skip=skip)
    value, bound = embed_reference(ids, g, vocab, scale, skip, grad.dtype)
    assert ((grad.double() - value).abs() <= bound).all()
    return g, grad


def draw_ids(n, vocab, seed=0, dtype=torch.int32, skew=4.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (vocab * torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) ** skew).long().clamp(max=vocab - 1).to(dtype)


@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 1000, 64), (7, 50, 13), (300, 999, 1000), (48, 3, 2048), (1000, 5000, 4104), (5, 10, 8200)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_forward(n, vocab, d, dtype):
    table = torch.randn(vocab, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).to(DT[dtype])
    forward(draw_ids(n, vocab), table, 1.0)
    forward(draw_ids(n, vocab, dtype=torch.int64), table, d ** 0.5)


def test_forward_of_ids_outside_the_table_strides_and_infinities():
    table = torch.randn(20, 72, device="cuda")[:, :65].bfloat16()  # odd rows
    ids = torch.tensor([0, -1, 19, 20, 2**31 - 1, -2**31, 3, 3], device="cuda", dtype=torch.int32)
    forward(ids, table, 2.0)
    wide = torch.randn(20, 80, device="cuda").bfloat16()
    out = torch.full((8, 100), float("nan"), device="cuda", dtype=torch.bfloat16)
    forward(ids, wide[:, :72], 0.5, out=out[:, 8:80])
    assert torch.isnan(out[:, :8]).all() and torch.isnan(out[:, 80:]).all()
    wide[3, 5], wide[19, 1] = float("nan"), float("inf")
    out = torch.empty(8, 80, device="cuda", dtype=torch.bfloat16)
    L.lapsum_embed_forward(ids.long(), wide, out, scale=0.0)  # zeros beside the rows that are not finite
    assert torch.isnan(out[6, 5]) and torch.isnan(out[2, 1]) and not out[[0, 1, 3, 4, 5]].any()


@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 700, 40), (31, 5, 8), (33, 1, 24), (64, 2, 64), (1000, 513, 130), (4093, 50021, 96), (20000, 512, 64),
                                       (9000, 1025, 2056)])
@pytest.mark.parametrize("dtype,wide", [("bf16", False), ("f16", True), ("f32", False)])
def test_backward(n, vocab, d, dtype, wide):
    backward(draw_ids(n, vocab, seed=n), vocab, d, dtype, scale=1.5, wide=wide)


@pytest.mark.parametrize("count", [15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 97, 4096])
def test_rows_of_many_positions_wherever_their_pieces_begin(count):
    for before in (0, 1, 15, 16, 31, 32, 40):
        ids = torch.cat([torch.arange(before), torch.full((count,), 50), torch.arange(51, 60)]).to(torch.int32)
        ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(count))].cuda()
        backward(ids, 64, 24, "f32")


def test_padding_ids_outside_and_neighbouring_long_rows():
    n = 5000
    ids = draw_ids(n, 40, seed=2, skew=1.0)   # every row is long
    ids[::7] = 11
    ids[::13] = -1
    ids[::17] = 40
    backward(ids, 40, 72, "bf16", skip=11)
    backward(ids.long(), 40, 72, "bf16", skip=11, wide=True)
    _, grad = backward(torch.full((100,), 5, device="cuda", dtype=torch.int32), 9, 16, "f32", skip=5)
    assert not grad.any()
    big = torch.tensor([2**40, 3, -2**40], device="cuda")
    backward(big, 9, 16, "f32")


def test_strides_scale_and_one_workspace_for_fewer_ids():
    ws = L.EmbedWorkspace(3000, 300, 56)
    for n in (3000, 1, 40, 2999):
        backward(draw_ids(n, 300, seed=n), 300, 56, "bf16", scale=-0.25, ws=ws, stride=61, seed=n)


def test_no_ids():
    ws = L.EmbedWorkspace(8, 30, 16)
    grad = torch.full((30, 16), 3.0, device="cuda")
    e = torch.empty(0, 16, device="cuda")
    L.lapsum_embed_backward(e, torch.empty(0, device="cuda", dtype=torch.int32), grad, ws)
    assert not grad.any()
    L.lapsum_embed_forward(torch.empty(0, device="cuda", dtype=torch.int32), grad, e)


def test_results_do_not_depend_on_scheduling():
    ids = draw_ids(20000, 3000, seed=8)
    first = backward(ids, 3000, 256, "bf16", wide=True)[1]
    for _ in range(3):
        assert torch.equal(first, backward(ids, 3000, 256, "bf16", wide=True)[1])


def test_gradient_against_differences():
    """the loss <g, out> is linear in the table: a step of 1 in one entry changes it by the gradient"""
    ids = torch.tensor([2, 0, 2, 1, 2], device="cuda", dtype=torch.int32)
    table = torch.randint(-4, 5, (4, 8), device="cuda").float()
    g, grad = backward(ids, 4, 8, "f32", scale=3.0)
    out = torch.empty(5, 8, device="cuda")

    def loss(t):
        L.lapsum_embed_forward(ids, t, out, scale=3.0)
        return (g.double() * out.double()).sum().item()

    for v in range(4):
        up = table.clone()
        up[v, 3] += 1
        assert abs(loss(up) - loss(table) - grad[v, 3].item()) <= 1e-5
