"""The dense operators under CUDA graphs, on streams of their own, with offsets beyond 32 bits, and what they refuse."""
import ctypes as C

import pytest
import torch

import paper_2608_06912_b200 as L
from tests.dense_util import sample_reference

pytestmark = pytest.mark.gpu


class Step:
    """one pass of every operator on buffers of its own"""

    def __init__(self, rows=96, n=264, k=136, vocab=1003, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = torch.bfloat16

        def rand(*shape, dt=bf):
            return torch.randn(*shape, device="cuda", generator=g).to(dt)

        self.ids = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
        self.table, self.x = rand(vocab, k), torch.empty(rows, k, device="cuda", dtype=bf)
        self.w, self.b, self.head = rand(n, k) * k ** -0.5, rand(n), rand(vocab, n) * n ** -0.5
        self.h, self.logits = torch.empty(rows, n, device="cuda", dtype=bf), torch.empty(rows, vocab, device="cuda")
        self.u, self.token, self.logprob = torch.rand(rows, device="cuda", generator=g), *(torch.empty(rows, device="cuda", dtype=t) for t in (torch.int32, torch.float32))
        self.ws1 = L.LinearWorkspace(rows, n, k, activation=L.ACT_SILU, training=True)
        self.ws2 = L.LinearWorkspace(rows, vocab, n, out_dtype=L.IO_F32, training=True)
        self.wse, self.pre = L.EmbedWorkspace(rows, vocab, k), self.ws1.new_pre()
        self.gl = rand(rows, vocab, dt=torch.float32)
        self.gh, self.gx = torch.empty_like(self.h), torch.empty_like(self.x)
        self.ghead, self.gw, self.gb = torch.empty_like(self.head, dtype=torch.float32), torch.empty_like(self.w), torch.empty_like(self.b)
        self.gt = torch.empty_like(self.table, dtype=torch.float32)

    def run(self, stream=None):
        L.lapsum_embed_forward(self.ids, self.table, self.x, scale=2.0, stream=stream)
        L.lapsum_linear_forward(self.x, self.w, self.b, None, self.h, self.ws1, pre=self.pre, stream=stream)
        L.lapsum_linear_forward(self.h, self.head, None, None, self.logits, self.ws2, stream=stream)
        L.lapsum_sample(self.logits, self.u, L.sample_params(top_p=0.9, top_k=50), self.token, self.logprob, stream=stream)
        L.lapsum_linear_backward(self.gl, self.h, self.head, None, self.gh, self.ghead, None, self.ws2, stream=stream)
        L.lapsum_linear_backward(self.gh, self.x, self.w, self.pre, self.gx, self.gw, self.gb, self.ws1, stream=stream)
        L.lapsum_embed_backward(self.gx, self.ids, self.gt, self.wse, scale=2.0, skip=3, stream=stream)

    def results(self):
        return [t.clone() for t in (self.h, self.logits, self.token, self.logprob, self.gh, self.ghead, self.gx, self.gw, self.gb, self.gt)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_captured_step_replays_with_new_inputs():
    s = Step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in (1, 2):
        other = Step(seed=seed)
        for name in ("ids", "table", "w", "b", "head", "u", "gl"):
            getattr(s, name).copy_(getattr(other, name))
        for t in (s.x, s.h, s.logits, s.gh, s.gx, s.ghead, s.gw, s.gb, s.gt):
            t.fill_(float("nan"))
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert same(s.results(), other.results())
    assert s.ws1.status() == 0 and s.ws2.status() == 0


def test_streams_given_and_current_at_the_same_time():
    want = []
    for seed in range(3):
        s = Step(seed=seed)
        s.run()
        torch.cuda.synchronize()
        want.append(s.results())
    steps = [Step(seed=seed) for seed in range(3)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(steps, streams):
            s.run(stream=st)
    torch.cuda.synchronize()
    assert all(same(s.results(), w) for s, w in zip(steps, want))
    with torch.cuda.stream(streams[0]):
        steps[1].run()
    torch.cuda.synchronize()
    assert same(steps[1].results(), want[1])


def test_back_to_back_calls_that_overlap_see_each_other_s_results():
    """every kernel may start while the one before it drains: a long chain of small calls that depend on each other"""
    rows, n = 40, 128
    g = torch.Generator(device="cuda").manual_seed(0)
    w = (torch.randn(n, n, device="cuda", generator=g) * n ** -0.5).bfloat16()
    a, b = (torch.randn(rows, n, device="cuda", generator=g).bfloat16() for _ in range(2))
    ws = L.LinearWorkspace(rows, n, n)
    outs = []
    for _ in range(2):
        x, y = a.clone(), b.clone()
        for _ in range(100):
            L.lapsum_linear_forward(x, w, None, y, y, ws)
            L.lapsum_linear_forward(y, w, None, None, x, ws)
        outs.append((x, y))
    x, y = a.clone(), b.clone()
    for _ in range(100):
        L.lapsum_linear_forward(x, w, None, y, y, ws)
        torch.cuda.synchronize()
        L.lapsum_linear_forward(y, w, None, None, x, ws)
        torch.cuda.synchronize()
    assert all(torch.equal(o[0], x) and torch.equal(o[1], y) for o in outs)


@pytest.mark.parametrize("rows,n,k", [(48, 1000, 512), (600, 600, 256), (4096, 2048, 512), (16, 128, 4096), (1021, 2048, 5632)])
def test_waits_that_run_out_end_with_a_status(rows, n, k):
    ws = L.LinearWorkspace(rows, n, k)
    x, w, y = (torch.zeros(*s, device="cuda", dtype=torch.bfloat16) for s in ((rows, k), (n, k), (rows, n)))
    rc = L.lib().lapsum_debug_linear_timeout(200, x.data_ptr(), w.data_ptr(), y.data_ptr(), C.byref(ws.dims), ws.ptr, ws.bytes,
                                             torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and ws.status() == L.ST_LINEAR_TIMEOUT
    fresh = L.LinearWorkspace(rows, n, k)  # the next call works
    L.lapsum_linear_forward(x, w, None, None, y, fresh)
    assert fresh.status() == 0 and not y.any()


def test_offsets_beyond_32_bits():
    bf = torch.bfloat16
    rows, n, k = 70001, 40000, 64   # 2.8e9 outputs
    x, w = torch.randn(rows, k, device="cuda").to(bf), torch.randn(n, k, device="cuda").to(bf)
    y = torch.empty(rows, n, device="cuda", dtype=bf)
    L.lapsum_linear_forward(x, w, None, None, y, L.LinearWorkspace(rows, n, k))
    for r in (0, 53000, 70000):
        want = x[r].double() @ w.double().t()
        assert ((y[r].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16).all()
    rows, vocab = 70001, 40000
    u = torch.rand(rows, device="cuda")
    token, kept = (torch.empty(rows, device="cuda", dtype=torch.int32) for _ in range(2))
    L.lapsum_sample(y, u, L.sample_params(top_k=7, io_dtype=L.IO_BF16), token, None, kept)
    at = [0, 53699, 70000]
    t, _, c = sample_reference(y[at], u[at].cpu(), [1.0] * 3, [7] * 3, [1.0] * 3, [0.0] * 3)
    assert token[at].tolist() == list(t) and kept[at].tolist() == list(c) and (kept == 7).all()
    del y
    vocab, d = 1_100_003, 2048     # 2.25e9 entries
    table = torch.empty(vocab, d, device="cuda", dtype=bf).normal_()
    ids = torch.tensor([0, 1_100_002, 1_048_577, 5, 1_100_002], device="cuda")
    out = torch.empty(5, d, device="cuda", dtype=bf)
    L.lapsum_embed_forward(ids, table, out)
    assert torch.equal(out, table[ids])
    table.fill_(1.0)
    L.lapsum_embed_backward(out, ids, table, L.EmbedWorkspace(5, vocab, d))
    assert torch.equal(table[1_100_002], (out[1].float() + out[4].float()).to(bf)) and torch.equal(table[1_048_577], out[2])
    assert int((table[::1000] != 0).any(1).sum()) <= 1 and not table[1_100_001].any()


def test_tensors_that_do_not_fit_are_refused():
    ws = L.LinearWorkspace(8, 24, 16, activation=L.ACT_RELU, training=True)
    bf = torch.bfloat16
    x, w, y = (torch.zeros(*s, device="cuda", dtype=bf) for s in ((8, 16), (24, 16), (8, 24)))
    pre = ws.new_pre()
    ok = dict(x=x, w=w, bias=None, residual=None, y=y, ws=ws, pre=pre)
    L.lapsum_linear_forward(**ok)
    for change, error in ((dict(x=x.half()), TypeError), (dict(x=x.cpu()), TypeError), (dict(x=torch.zeros(9, 16, device="cuda", dtype=bf)), ValueError),
                          (dict(x=x[:, :8]), ValueError), (dict(w=w.t().contiguous()), ValueError), (dict(w=w[:, ::2]), TypeError),
                          (dict(bias=torch.zeros(23, device="cuda", dtype=bf)), ValueError), (dict(bias=torch.zeros(24, device="cuda", dtype=torch.half)), TypeError),
                          (dict(residual=y.float()), TypeError), (dict(residual=y[:7]), ValueError), (dict(y=y.t()), TypeError),
                          (dict(pre=None), TypeError), (dict(pre=pre[:4]), ValueError), (dict(pre=y), TypeError),
                          (dict(x=torch.zeros(8 * 18, device="cuda", dtype=bf)[8:].as_strided((8, 16), (17, 1))), L.LapsumError)):
        with pytest.raises(error):
            L.lapsum_linear_forward(**{**ok, **change})
    with pytest.raises(ValueError):
        L.LinearWorkspace(8, 24, 16).new_pre()
    with pytest.raises(L.LapsumError):
        L.LinearWorkspace(8, 24, 17)
    with pytest.raises(L.LapsumError):  # not a training workspace
        L.lapsum_linear_backward(y, x, w, None, None, None, None, L.LinearWorkspace(8, 24, 16))
    logits, u, token = torch.zeros(3, 9, device="cuda"), torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.int32)
    for kw, error in ((dict(u=u[:2]), ValueError), (dict(u=u.double()), TypeError), (dict(token=token.long()), TypeError), (dict(logits=logits.t()), TypeError),
                      (dict(temperature=u[:2]), ValueError), (dict(top_k=u), TypeError), (dict(logits=logits.half()), TypeError)):
        with pytest.raises(error):
            L.lapsum_sample(**{**dict(logits=logits, u=u, params=L.sample_params(), token=token), **kw})
    table, ids, out = torch.zeros(5, 8, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.int32), torch.zeros(3, 8, device="cuda")
    for args, error in (((ids.short(), table, out), TypeError), ((ids, table.double(), out.double()), TypeError), ((ids, table, out[:2]), ValueError),
                        ((ids[:, None], table, out), TypeError), ((ids, table, out.half()), TypeError)):
        with pytest.raises(error):
            L.lapsum_embed_forward(*args)
    es = L.EmbedWorkspace(3, 5, 8)
    with pytest.raises(ValueError):
        L.lapsum_embed_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.int32), table, es)
    with pytest.raises(TypeError):
        L.lapsum_embed_backward(out.half(), ids, table.bfloat16(), es)
