"""The experts' products and their gradients against 64 bits (bounds: tests/experts_util.py), and their refusals."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import chosen, experts_reference

pytestmark = pytest.mark.gpu


class Run:
    def __init__(self, T, E, k, d, f, dtype=torch.bfloat16, training=False, seed=0, drop=0.0, idx=None, tile_rows=None, skew=0.7,
                 pad=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gen = gen

        def rand(*shape, scale=1.0):
            return (scale * torch.randn(*shape, device="cuda", generator=gen)).to(dtype)

        self.x = rand(T, d + pad)[:, :d]
        self.a, self.b = rand(E, 2 * f, d, scale=d ** -0.5), rand(E, d, f, scale=f ** -0.5)
        self.idx = chosen(T, E, k, gen, drop, skew) if idx is None else idx.to("cuda", torch.int32)
        self.w = torch.rand(T, k, device="cuda", generator=gen) + 0.05
        self.gy = rand(T, d + pad)[:, :d]
        self.training = training
        self.disp = L.Dispatch(T, k, E, tile_rows=tile_rows, training=training)
        self.ws = L.ExpertsWorkspace(self.disp, d, f, io_dtype=L.IO_OF[dtype], training=training)
        self.saved = self.ws.new_saved() if training else None
        if training:
            self.saved.fill_(255)  # NaN bytes: nothing may rely on what a buffer held
        self.disp.buf.fill_(255)
        self.ws.buf[256:].fill_(255)

    def __call__(self, stream=None):
        nan = lambda t, dtype=None: torch.full(t.shape, float("nan"), device="cuda", dtype=dtype or t.dtype)  # noqa: E731
        self.out = {"y": nan(self.x)}
        L.lapsum_dispatch(self.idx, self.disp, stream)
        L.lapsum_experts_forward(self.x, self.a, self.b, self.w, self.disp, self.out["y"], self.ws, saved=self.saved, stream=stream)
        if self.training:
            self.out.update(grad_x=nan(self.x), grad_w_gate_up=nan(self.a), grad_w_down=nan(self.b), grad_w=nan(self.w, self.x.dtype))
            o = self.out
            L.lapsum_experts_backward(self.gy, self.x, self.a, self.b, self.w, self.disp, self.saved, o["grad_x"], o["grad_w_gate_up"],
                                      o["grad_w_down"], o["grad_w"], self.ws, stream=stream)
        return self.out

    def check(self):
        out = self()
        torch.cuda.synchronize()
        assert self.ws.status() == 0
        ref = experts_reference(self.x, self.a, self.b, self.idx, self.w, self.gy if self.training else None)
        for name, (want, bound) in ref.items():
            got = out[name].double()
            assert torch.isfinite(got).all(), name
            worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
            assert worst <= 1.0, f"{name}: {worst:.3f} of the bound"


@pytest.mark.parametrize("T", [1, 2, 7, 64, 333])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_forward(T, dtype):
    Run(T, 12, 3, 200, 136, dtype, seed=T).check()


@pytest.mark.parametrize("T,k", [(1, 1), (1, 8), (2, 3), (4, 32)])
@pytest.mark.parametrize("d,f", [(8, 8), (1000, 520), (2048, 1024), (2056, 2056), (4104, 4104), (72, 5000)])
def test_few_tokens(T, k, d, f):
    """no tensor core: rows shorter and longer than a stage, several choices' rows in a stage, dropped entries"""
    Run(T, 33, k, d, f, seed=T + d).check()
    Run(T, 33, k, d, f, torch.float16, seed=T + d, drop=0.5).check()


@pytest.mark.parametrize("rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d,f", [(8, 8), (64, 64), (72, 40), (256, 128), (520, 264), (1000, 1032)])
def test_forward_on_every_row_tile(rows, d, f):
    Run(150, 5, 2, d, f, tile_rows=rows, seed=rows + d).check()


@pytest.mark.parametrize("T,E,k,d,f", [
    (1, 4, 1, 64, 64), (3, 4, 4, 72, 40), (40, 6, 2, 128, 264), (257, 3, 2, 328, 200), (600, 5, 3, 256, 512), (130, 40, 1, 136, 72),
])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_training(T, E, k, d, f, dtype):
    Run(T, E, k, d, f, dtype, training=True, seed=T + d).check()


@pytest.mark.parametrize("rows", [64, 128, 256])
@pytest.mark.parametrize("d,f", [(192, 320), (72, 40), (520, 264)])
def test_training_on_every_row_tile(rows, d, f):
    Run(300, 7, 2, d, f, training=True, tile_rows=rows, seed=5).check()


@pytest.mark.parametrize("rows", [64, 128, 256])
def test_training_with_more_tiles_than_processors(rows):
    """every block walks over several tiles, in both accumulators and round the ring"""
    Run(3000, 16, 4, 512, 768, training=True, tile_rows=rows, seed=6).check()


def test_dropped_entries_and_tokens_without_any():
    gen = torch.Generator(device="cuda").manual_seed(3)
    idx = chosen(90, 9, 3, gen, drop=0.4)
    idx[5:20] = -1          # tokens without an expert
    idx[21, 0] = 9          # beyond the experts: dropped like -1
    idx[22, 1] = 2 ** 31 - 1
    idx[23, 2] = -2 ** 31
    idx[idx == 4] = -1      # an expert without a token
    r = Run(90, 9, 3, 104, 88, training=True, idx=idx, seed=4)
    r.check()
    assert (r.out["y"][5:20] == 0).all() and (r.out["grad_x"][5:20] == 0).all()
    assert (r.out["grad_w"][5:20] == 0).all() and (r.out["grad_w_gate_up"][4] == 0).all() and (r.out["grad_w_down"][4] == 0).all()


def test_nothing_routed():
    r = Run(33, 6, 2, 64, 72, training=True, idx=torch.full((33, 2), -1), seed=1)
    r.check()
    assert all((v == 0).all() for v in r.out.values())


def test_all_tokens_to_one_expert_on_narrow_tiles():
    Run(500, 64, 1, 136, 72, idx=torch.full((500, 1), 41), tile_rows=16, seed=2).check()


@pytest.mark.parametrize("rows", [16, 32, 64])
def test_wide_column_tiles_on_narrow_row_tiles(rows):
    Run(200, 60, 4, 264, 1032, tile_rows=rows, seed=3).check()  # enough tiles for 256 columns


def test_an_expert_twice_for_one_token():
    Run(20, 4, 2, 64, 64, training=True, idx=torch.full((20, 2), 3), seed=2).check()


def test_rows_of_x_and_grad_y_may_be_strided():
    Run(70, 5, 2, 88, 96, training=True, pad=24, seed=6).check()


def test_no_tokens():
    r = Run(0, 5, 2, 64, 72, training=True, idx=torch.zeros(0, 2))
    out = r()
    torch.cuda.synchronize()
    assert out["y"].shape == (0, 64) and (out["grad_w_gate_up"] == 0).all() and (out["grad_w_down"] == 0).all()


def test_infinite_weights_of_one_expert_stay_with_its_tokens():
    r = Run(60, 4, 1, 72, 80, training=True, idx=(torch.arange(60) % 4).view(60, 1), seed=8)
    r.a[2, 3] = float("inf")
    r.b[2, 5] = float("nan")
    out = r()
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    sound = (r.idx[:, 0] != 2)
    for name in ("y", "grad_x", "grad_w"):
        want, bound = ref[name]
        assert torch.isfinite(out[name][sound]).all(), name
        assert ((out[name].double() - want).abs()[sound] <= bound[sound]).all(), name
    for name in ("grad_w_gate_up", "grad_w_down"):
        want, bound = ref[name]
        for e in (0, 1, 3):
            assert ((out[name][e].double() - want[e]).abs() <= bound[e]).all(), name


def test_the_same_bits_again_and_on_another_stream():
    r = Run(400, 8, 2, 264, 136, training=True, seed=9)
    first = {n: v.clone() for n, v in r().items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = r(stream=side)
    side.synchronize()
    for n in first:
        assert torch.equal(first[n], second[n]), n


def test_gradients_against_differences():
    """<gradient, direction> against central differences of the 64-bit forward; the bound is the elements' bounds along the direction
    (independent errors), the differences' own error (about step^2) is far below it"""
    r = Run(40, 4, 2, 64, 72, torch.float16, training=True, seed=11)
    out = r()
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    args = {"grad_x": r.x.double(), "grad_w_gate_up": r.a.double(), "grad_w_down": r.b.double(), "grad_w": r.w.double()}

    def loss(x, a, b, w):
        y = torch.zeros_like(x)
        for e in range(a.shape[0]):
            t, j = (r.idx == e).nonzero(as_tuple=True)
            g, u = (x[t] @ a[e].T).chunk(2, 1)
            y.index_add_(0, t, w[t, j][:, None] * ((g * torch.sigmoid(g) * u) @ b[e].T))
        return (y * r.gy.double()).sum()

    order = ["grad_x", "grad_w_gate_up", "grad_w_down", "grad_w"]
    for name in order:
        direction = torch.randn(args[name].shape, device="cuda", dtype=torch.float64, generator=r.gen)
        step = 1e-4
        hi, lo = [loss(*[args[n] + (s * step * direction if n == name else 0) for n in order]) for s in (1, -1)]
        want = ((hi - lo) / (2 * step)).item()
        got = (out[name].double() * direction).sum().item()
        bound = 2 * ((ref[name][1] * direction) ** 2).sum().sqrt().item()
        assert abs(got - want) <= bound, (name, got, want, bound)


def test_offsets_beyond_32_bits():
    """1.12 million slots of 2048 columns: more than 2^31 elements per slot buffer; a sample of the tokens is checked"""
    T, E, k, d, f = 140_000, 16, 8, 2048, 64
    r = Run(T, E, k, d, f, seed=14, tile_rows=128)
    assert r.disp.capacity * d > 2 ** 31
    out = r()
    torch.cuda.synchronize()
    assert r.ws.status() == 0
    late = torch.cat([torch.arange(64), torch.randint(0, T, (128,)), torch.arange(T - 64, T)]).cuda()
    want, bound = experts_reference(r.x[late], r.a, r.b, r.idx[late], r.w[late])["y"]
    assert ((out["y"][late].double() - want).abs() <= bound).all()


def test_cuda_graph_replay():
    r = Run(64, 8, 2, 128, 64, training=True, seed=12)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = r()
    fresh = torch.randn_like(r.x)
    r.x.copy_(fresh)
    r.idx.copy_(chosen(64, 8, 2, r.gen))
    graph.replay()
    torch.cuda.synchronize()
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    for name, (want, bound) in ref.items():
        assert ((out[name].double() - want).abs() <= bound).all(), name


def test_a_wait_that_runs_out_is_reported():
    import ctypes as C

    r = Run(8, 4, 2, 64, 64)
    L.lapsum_dispatch(r.idx, r.disp)
    rc = L.lib().lapsum_debug_experts_timeout(1000, r.ws.ptr, r.ws.bytes, r.disp.ptr, r.disp.bytes, r.x.data_ptr(), r.a.data_ptr(),
                                              r.w.data_ptr(), C.byref(r.ws.dims), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert r.ws.status() == L.ST_EXPERTS_TIMEOUT
    out = r()  # the context is usable; the workspace keeps the bit until it is made again
    torch.cuda.synchronize()
    want, bound = experts_reference(r.x, r.a, r.b, r.idx, r.w)["y"]
    assert ((out["y"].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("T,training", [(3, False), (40, False), (300, True)])
def test_tables_of_another_batch_s_bytes_do_no_harm(T, training):
    """Tables that hold anything (a dispatch that was forgotten): the results mean nothing, but every index is checked, so the call
    ends and the workspace serves the next batch"""
    r = Run(T, 6, 2, 72, 80, training=training, seed=15)
    dispatch = L.lapsum_dispatch
    gen = torch.Generator(device="cuda").manual_seed(16)
    for low, high in ((-2 ** 31, 2 ** 31 - 1), (-5, 4000), (0, 7)):
        words = r.disp.buf.view(torch.int32)
        words.copy_(torch.randint(low, high, words.shape, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32))
        try:
            L.lapsum_dispatch = lambda *a: None
            r()
        finally:
            L.lapsum_dispatch = dispatch
        torch.cuda.synchronize()
    r.check()


def test_refusals():
    r = Run(8, 4, 2, 64, 64, training=True)
    o = torch.empty_like(r.x)
    L.lapsum_dispatch(r.idx, r.disp)
    fwd = lambda **kw: L.lapsum_experts_forward(**{**dict(x=r.x, w_gate_up=r.a, w_down=r.b, w=r.w, dispatch=r.disp, y=o, ws=r.ws,  # noqa: E731
                                                          saved=r.saved), **kw})
    fwd()
    for bad, exc in ((dict(x=r.x.float()), TypeError), (dict(x=r.x.cpu()), TypeError), (dict(x=r.x.t().contiguous().t()), TypeError),
                     (dict(x=r.x[:4]), ValueError), (dict(w_gate_up=r.a[:2]), ValueError), (dict(w_down=r.b.half()), TypeError),
                     (dict(w=r.w.half()), TypeError), (dict(y=o[:, :32]), TypeError), (dict(saved=None), L.LapsumError),
                     (dict(saved=r.saved[:256]), L.LapsumError), (dict(dispatch=L.Dispatch(8, 2, 4, tile_rows=128)), ValueError)):
        with pytest.raises(exc):
            fwd(**bad)
    raw = torch.empty(r.x.numel() + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(L.LapsumError):  # not at a multiple of 16 bytes
        fwd(x=raw[1:1 + r.x.numel()].view(8, 64))
    with pytest.raises(L.LapsumError):  # row stride no multiple of 8
        fwd(x=torch.empty(8, 67, dtype=torch.bfloat16, device="cuda")[:, :64])
    for d, f in ((60, 64), (64, 60), (0, 64)):
        with pytest.raises(L.LapsumError):
            L.ExpertsWorkspace(r.disp, d, f, training=True)
    with pytest.raises(L.LapsumError):
        L.ExpertsWorkspace(r.disp, 64, 64, io_dtype=L.IO_F32)
    with pytest.raises(L.LapsumError):  # training needs row tiles of 64 or 128
        L.ExpertsWorkspace(L.Dispatch(8, 2, 4, tile_rows=16), 64, 64, training=True)
    serving = Run(8, 4, 2, 64, 64)
    with pytest.raises(ValueError):
        serving.ws.new_saved()
    with pytest.raises(L.LapsumError):  # no backward on a serving workspace
        L.lapsum_experts_backward(r.gy, r.x, r.a, r.b, r.w, serving.disp, r.saved, o, torch.empty_like(r.a), torch.empty_like(r.b),
                                  torch.empty(8, 2, dtype=torch.bfloat16, device="cuda"), serving.ws)
