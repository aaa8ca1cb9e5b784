"""A model's step made of all operators: embed, a dense layer, the router and its experts, the vocabulary's logits, the next token; and its gradients
back to the table, against automatic differentiation in 64 bits with the same choice of experts."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import sample_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,vocab,d,f,E,k", [(1, 300, 64, 96, 4, 2), (37, 1003, 136, 200, 8, 2), (300, 2000, 256, 128, 16, 4)])
def test_a_step_and_its_gradients(tokens, vocab, d, f, E, k):
    bf, gen = torch.bfloat16, torch.Generator(device="cuda").manual_seed(tokens)

    def rand(*shape, scale=1.0):
        return (scale * torch.randn(*shape, device="cuda", generator=gen)).to(bf)

    def new(*shape, dt=bf):
        return torch.empty(*shape, device="cuda", dtype=dt)

    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    table, w1, b1, wr = rand(vocab, d), rand(d, d, scale=d ** -0.5), rand(d, scale=0.1), rand(E, d, scale=d ** -0.5)
    wgu, wd, head = rand(E, 2 * f, d, scale=d ** -0.5), rand(E, d, f, scale=f ** -0.5), rand(vocab, d, scale=d ** -0.5)
    # forward
    x, h, y, r = new(tokens, d), new(tokens, d), new(tokens, d), new(tokens, E, dt=torch.float32)
    logits = new(tokens, vocab, dt=torch.float32)
    idx, wts = new(tokens, k, dt=torch.int32), new(tokens, k, dt=torch.float32)
    dense = L.LinearWorkspace(tokens, d, d, activation=L.ACT_GELU, training=True)
    router = L.LinearWorkspace(tokens, E, d, out_dtype=L.IO_F32, training=True)
    last = L.LinearWorkspace(tokens, vocab, d, out_dtype=L.IO_F32, training=True)
    tables = L.Dispatch(tokens, k, E, training=True)
    experts = L.ExpertsWorkspace(tables, d, f, training=True)
    pre, saved, rp = dense.new_pre(), experts.new_saved(), L.route_params(k=k)
    L.lapsum_embed_forward(ids, table, x, scale=0.5)
    L.lapsum_linear_forward(x, w1, b1, x, h, dense, pre=pre)
    L.lapsum_linear_forward(h, wr, None, None, r, router)
    L.lapsum_route_forward(r, None, rp, idx, wts)
    L.lapsum_dispatch(idx, tables)
    L.lapsum_experts_forward(h, wgu, wd, wts, tables, y, experts, saved=saved)
    L.lapsum_linear_forward(y, head, None, None, logits, last)
    u, token, kept = torch.rand(tokens, device="cuda", generator=gen), new(tokens, dt=torch.int32), new(tokens, dt=torch.int32)
    logprob = new(tokens, dt=torch.float32)
    L.lapsum_sample(logits, u, L.sample_params(temperature=0.7, top_k=40, top_p=0.9), token, logprob, kept)
    # backward of the sum of log probabilities' gradient-like upstream
    gl = torch.randn(tokens, vocab, device="cuda", generator=gen)
    gy, gh, gx, gr = new(tokens, d), new(tokens, d), new(tokens, d), new(tokens, E, dt=torch.float32)
    gh_r, gwts = new(tokens, d), new(tokens, k, dt=torch.float32)
    g_head, g_gu, g_d = new(vocab, d, dt=torch.float32), torch.empty_like(wgu), torch.empty_like(wd)
    g_r, g_w1, g_b1, g_table = new(E, d, dt=torch.float32), new(d, d), new(d), new(vocab, d, dt=torch.float32)
    L.lapsum_linear_backward(gl, y, head, None, gy, g_head, None, last)
    L.lapsum_experts_backward(gy, h, wgu, wd, wts, tables, saved, gh, g_gu, g_d, gwts, experts)
    L.lapsum_route_backward(gwts, r, idx, wts, rp, gr)
    L.lapsum_linear_backward(gr, h, wr, None, gh_r, g_r, None, router)
    gh += gh_r
    L.lapsum_linear_backward(gh, x, w1, pre, gx, g_w1, g_b1, dense)
    gx += gh  # the residual's
    L.lapsum_embed_backward(gx, ids, g_table, L.EmbedWorkspace(tokens, vocab, d), scale=0.5)
    assert dense.status() == router.status() == last.status() == experts.status() == 0
    # 64 bits
    p = [t.double().requires_grad_() for t in (table, w1, b1, wr, wgu, wd, head)]
    x64 = 0.5 * p[0][ids.long()]
    h64 = torch.nn.functional.gelu(x64 @ p[1].t() + p[2]) + x64
    chosen = torch.softmax((h64 @ p[3].t()).gather(1, idx.long()), 1)
    y64 = 0
    for j in range(k):
        e = idx[:, j].long()
        gate, up = torch.einsum("tfd,td->tf", p[4][e], h64).chunk(2, 1)
        y64 = y64 + chosen[:, j:j + 1] * torch.einsum("tdf,tf->td", p[5][e], torch.nn.functional.silu(gate) * up)
    l64 = y64 @ p[6].t()
    want = torch.autograd.grad(l64, p, gl.double())
    # seven roundings of 2^-9 on the way there, some fifteen back, each at most doubled by a step's slope, as independent errors
    assert (logits.double() - l64).norm() <= 4 * 7 ** 0.5 * 2.0 ** -9 * l64.norm()
    for got, ref in zip((g_table, g_w1, g_b1, g_r, g_gu, g_d, g_head), want):
        assert (got.double() - ref).norm() <= 4 * 22 ** 0.5 * 2.0 ** -9 * ref.norm()
    t, lp, n = sample_reference(logits, u.cpu(), [0.7] * tokens, [40] * tokens, [0.9] * tokens, [0.0] * tokens)
    # 0.7 and 0.9 are doubles for all rows here and there
    assert token.tolist() == list(t) and kept.tolist() == list(n)
