"""Streams and devices of the mixture-of-experts calls, on the host alone: CPU tensors that say they are on a GPU, and a library that
notes its calls."""
import contextlib

import pytest
import torch

import paper_2608_06912_b200 as L
from paper_2608_06912_b200 import experts as X


class Fake(torch.Tensor):
    """A CPU tensor that claims to be on a GPU and notes the streams it is recorded on (views share their base's notes)."""

    is_cuda = True
    notes, gpu = None, 0

    @property
    def device(self):
        return torch.device("cuda", self.gpu)

    def get_device(self):
        return self.gpu

    def record_stream(self, stream):
        self.notes.append(stream.cuda_stream)

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        out = super().__torch_function__(func, types, args, kwargs or {})
        if isinstance(out, Fake) and out.notes is None:
            src = next(a for a in args if isinstance(a, Fake))
            out.notes, out.gpu = src.notes, src.gpu
        return out


def fake(t, gpu=0):
    f = torch.Tensor._make_subclass(Fake, t)
    f.notes, f.gpu = [], gpu
    return f


class Stream:
    def __init__(self, handle, gpu=0):
        self.cuda_stream, self.device, self.device_index = handle, torch.device("cuda", gpu), gpu


class World:
    """one process with several GPUs: the current device, the current stream of each, and the calls that reached the library"""

    def __init__(self, monkeypatch):
        self.device, self.streams, self.calls, self.made = 0, {0: 0, 1: 0}, [], []
        real = L.lib()
        world = self

        class Lib:
            def __getattr__(self, name):
                if name in ("lapsum_route_default_params", "lapsum_dispatch_tile_rows", "lapsum_dispatch_describe", "lapsum_experts_describe"):
                    return getattr(real, name)
                return lambda *a: world.calls.append(name) or 0

        def buffer(n, device):
            raw = fake(torch.empty(n + 256, dtype=torch.uint8), device.index)
            world.made.append(world.streams[device.index])  # the allocator's memory belongs to the current stream
            return raw[-torch.Tensor.data_ptr(raw) % 256:][:n]

        @contextlib.contextmanager
        def on(stream):
            before = (self.device, dict(self.streams))
            if stream is not None:
                self.device, self.streams[stream.device_index] = stream.device_index, stream.cuda_stream
            try:
                yield
            finally:
                self.device, self.streams = before

        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(X, "lib", lambda: Lib())
        monkeypatch.setattr(X, "_buffer", buffer)
        monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.device)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.streams[i], raising=False)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(self.streams[self.device if d is None else torch.device(d).index]))


@pytest.fixture
def world(monkeypatch):
    return World(monkeypatch)


T, E, K, D, F = 8, 4, 2, 64, 72
BF16 = torch.bfloat16


def batch(gpu=0):
    """operands of a training step"""
    z = lambda *s, dt=BF16: fake(torch.zeros(*s, dtype=dt), gpu)  # noqa: E731
    return dict(idx=z(T, K, dt=torch.int32), x=z(T, D), a=z(E, 2 * F, D), b=z(E, D, F), w=z(T, K, dt=torch.float32), y=z(T, D), gy=z(T, D), gx=z(T, D),
                ga=z(E, 2 * F, D), gb=z(E, D, F), gw=z(T, K))


def step(o, disp, ws, saved, stream=None):
    L.lapsum_dispatch(o["idx"], disp, stream)
    L.lapsum_experts_forward(o["x"], o["a"], o["b"], o["w"], disp, o["y"], ws, saved=saved, stream=stream)
    L.lapsum_experts_backward(o["gy"], o["x"], o["a"], o["b"], o["w"], disp, saved, o["gx"], o["ga"], o["gb"], o["gw"], ws, stream=stream)


@pytest.mark.parametrize("how", ["current", "argument"])
def test_buffers_are_recorded_on_the_stream_that_a_call_uses(world, how):
    disp = L.Dispatch(T, K, E, training=True)
    ws = L.ExpertsWorkspace(disp, D, F, training=True)
    saved, o = ws.new_saved(), batch()
    step(o, disp, ws, saved)
    assert disp.buf.notes == [] and ws.buf.notes == []  # the stream that they were made on needs no record
    if how == "current":
        world.streams[0] = 1234  # `with torch.cuda.stream(side):`
        step(o, disp, ws, saved)
    else:
        step(o, disp, ws, saved, Stream(1234))
    assert set(disp.buf.notes) == {1234} and set(ws.buf.notes) == {1234}
    L.lapsum_dispatch(o["idx"], disp, Stream(99))  # every further stream
    assert set(disp.buf.notes) == {1234, 99}
    step(o, disp, ws, saved)
    ws.status(Stream(98))
    assert 98 in ws.buf.notes


def test_a_workspace_s_memory_belongs_to_the_stream_that_clears_it(world):
    """the allocator's memory may still be written by work queued on the stream that it is asked for on: a memset on another stream
    would not wait for that"""
    disp = L.Dispatch(T, K, E, training=True)
    ws = L.ExpertsWorkspace(disp, D, F, training=True, stream=Stream(77))
    assert world.made[-1] == 77 and ws.buf.notes == []
    saved, o = ws.new_saved(), batch()
    step(o, disp, ws, saved)  # on the current stream
    assert set(ws.buf.notes) == {0} and disp.buf.notes == []
    world.streams[0] = 55
    ws = L.ExpertsWorkspace(disp, D, F, training=True)
    assert world.made[-1] == 55 and ws.buf.notes == []


def route_operands(gpu=0):
    z = lambda *s, dt=torch.float32: fake(torch.zeros(*s, dtype=dt), gpu)  # noqa: E731
    return [z(T, E), z(E), L.route_params(k=K), z(T, K, dt=torch.int32), z(T, K)]


def back_operands(gpu=0):
    z = lambda *s, dt=torch.float32: fake(torch.zeros(*s, dtype=dt), gpu)  # noqa: E731
    return [z(T, K), z(T, E), z(T, K, dt=torch.int32), z(T, K), L.route_params(k=K), z(T, E)]


def refused(world, call):
    before = list(world.calls)
    with pytest.raises(ValueError, match="cuda:"):
        call()
    assert world.calls == before  # nothing reached the library


def test_tensors_of_several_devices_are_refused(world):
    disp = L.Dispatch(T, K, E, training=True)
    ws = L.ExpertsWorkspace(disp, D, F, training=True)
    saved, o = ws.new_saved(), batch()
    L.lapsum_route_forward(*route_operands())
    L.lapsum_route_backward(*back_operands())
    step(o, disp, ws, saved)
    for i in (1, 3, 4):
        args = route_operands()
        args[i] = route_operands(1)[i]
        refused(world, lambda: L.lapsum_route_forward(*args))
    for i in (0, 2, 3, 5):
        args = back_operands()
        args[i] = back_operands(1)[i]
        refused(world, lambda: L.lapsum_route_backward(*args))
    other = batch(1)
    refused(world, lambda: L.lapsum_dispatch(other["idx"], disp))
    fwd = dict(x=o["x"], w_gate_up=o["a"], w_down=o["b"], w=o["w"], dispatch=disp, y=o["y"], ws=ws, saved=saved)
    elsewhere = fake(torch.zeros(ws.saved_bytes, dtype=torch.uint8), 1)
    for name, key in (("x", "x"), ("w_gate_up", "a"), ("w_down", "b"), ("w", "w"), ("y", "y")):
        refused(world, lambda: L.lapsum_experts_forward(**{**fwd, name: other[key]}))
    refused(world, lambda: L.lapsum_experts_forward(**{**fwd, "saved": elsewhere}))
    back = dict(grad_y=o["gy"], x=o["x"], w_gate_up=o["a"], w_down=o["b"], w=o["w"], dispatch=disp, saved=saved, grad_x=o["gx"], grad_w_gate_up=o["ga"],
                grad_w_down=o["gb"], grad_w=o["gw"], ws=ws)
    L.lapsum_experts_backward(**back)
    for name, key in (("grad_y", "gy"), ("x", "x"), ("w_gate_up", "a"), ("w_down", "b"), ("w", "w"), ("grad_x", "gx"), ("grad_w_gate_up", "ga"),
                      ("grad_w_down", "gb"), ("grad_w", "gw")):
        refused(world, lambda: L.lapsum_experts_backward(**{**back, name: other[key]}))
    refused(world, lambda: L.lapsum_experts_backward(**{**back, "saved": elsewhere}))
    far = L.Dispatch(T, K, E, training=True, device="cuda:1")
    refused(world, lambda: L.lapsum_experts_forward(**{**fwd, "dispatch": far}))
    refused(world, lambda: L.lapsum_experts_backward(**{**back, "dispatch": far}))


def test_a_device_that_is_not_current_is_refused(world):
    """the launches go to the current device; another one's tensors would be foreign memory there"""
    disp = L.Dispatch(T, K, E, training=True, device="cuda:1")  # tables may be made for any device
    assert disp.device == torch.device("cuda", 1)
    refused(world, lambda: L.ExpertsWorkspace(disp, D, F, training=True))
    world.device = 1
    ws = L.ExpertsWorkspace(disp, D, F, training=True)
    saved, o = ws.new_saved(), batch(1)
    step(o, disp, ws, saved)
    ws.status()
    L.lapsum_route_forward(*route_operands(1))
    L.lapsum_route_backward(*back_operands(1))
    world.device = 0
    refused(world, lambda: L.lapsum_route_forward(*route_operands(1)))
    refused(world, lambda: L.lapsum_route_backward(*back_operands(1)))
    refused(world, lambda: L.lapsum_dispatch(o["idx"], disp))
    refused(world, lambda: L.lapsum_experts_forward(o["x"], o["a"], o["b"], o["w"], disp, o["y"], ws, saved=saved))
    refused(world, lambda: L.lapsum_experts_backward(o["gy"], o["x"], o["a"], o["b"], o["w"], disp, saved, o["gx"], o["ga"], o["gb"], o["gw"], ws))
    refused(world, lambda: ws.status())


def test_a_stream_of_another_device_is_refused(world):
    disp = L.Dispatch(T, K, E)
    ws = L.ExpertsWorkspace(disp, D, F)
    o, far = batch(), Stream(7, gpu=1)
    refused(world, lambda: L.lapsum_route_forward(*route_operands(), stream=far))
    refused(world, lambda: L.lapsum_dispatch(o["idx"], disp, far))
    refused(world, lambda: L.lapsum_experts_forward(o["x"], o["a"], o["b"], o["w"], disp, o["y"], ws, stream=far))
    refused(world, lambda: L.ExpertsWorkspace(disp, D, F, stream=far))
    refused(world, lambda: ws.status(far))


def test_the_weights_gradient_may_be_fp32(world):
    disp = L.Dispatch(T, K, E, training=True)
    ws = L.ExpertsWorkspace(disp, D, F, training=True)
    saved, o = ws.new_saved(), batch()
    wide = fake(torch.zeros(T, K), 0)
    L.lapsum_experts_backward(o["gy"], o["x"], o["a"], o["b"], o["w"], disp, saved, o["gx"], o["ga"], o["gb"], wide, ws)
    assert world.calls[-1] == "lapsum_experts_backward"
    import ctypes as C

    from paper_2608_06912_b200 import binding as B
    out, real = B.ExpertsLayout(), L.lib()
    for flag, rc in ((0, 0), (1, 0), (2, -7), (-1, -7)):
        d = B.ExpertsDims(tokens=T, experts=E, d=D, f=F, k=K, tile_rows=64, io_dtype=L.IO_BF16, training=1, grad_w_f32=flag)
        assert real.lapsum_experts_describe(C.byref(d), C.byref(out)) == rc, flag
