"""Binding of the mixture-of-experts entry points of include/lapsum.h: route, dispatch, experts.

    route     lapsum_route_forward / lapsum_route_backward    logits (or a soft mask) -> chosen experts and weights
    dispatch  Dispatch, lapsum_dispatch                       chosen experts -> tables that group the tokens by expert
    experts   ExpertsWorkspace, lapsum_experts_forward / lapsum_experts_backward

Argument marshalling only, like binding.py.  Outputs are the caller's tensors.  A call made on another stream than the
one its tensors were made on follows PyTorch's rules: the caller orders the streams, and records tensors of its own (`saved` among
them).  Buffers that Dispatch and ExpertsWorkspace own are recorded on the stream of every call, given or current, so
dropping the object early is safe.  A call's tensors are all on the current device, and so is its stream; anything else is refused.
"""
from __future__ import annotations

import ctypes as C
from contextlib import nullcontext
from typing import Optional

import torch

from . import binding as _b
from .binding import DispatchLayout, ExpertsDims, ExpertsLayout, IO_BF16, IO_F32, IO_TORCH, RouteParams, _check, lib

ROUTE_SOFTMAX, ROUTE_SIGMOID, ROUTE_GIVEN = 0, 1, 2
ROUTE_SCORES = {"softmax": ROUTE_SOFTMAX, "sigmoid": ROUTE_SIGMOID, "given": ROUTE_GIVEN}
IO_OF = {t: i for i, t in IO_TORCH.items()}


def route_params(**overrides) -> RouteParams:
    """lapsum_route_default_params with the named fields replaced."""
    p = RouteParams()
    lib().lapsum_route_default_params(C.byref(p))
    for key, val in overrides.items():
        if not hasattr(p, key):
            raise AttributeError(key)
        setattr(p, key, val)
    return p


def _stream(stream: Optional[torch.cuda.Stream], gpu: int) -> int:
    """The handle of a call's stream on the GPU of its tensors, which has to be the current one: the library launches there."""
    if torch._C._cuda_getDevice() != gpu:
        raise ValueError(f"the tensors are on cuda:{gpu}, but cuda:{torch._C._cuda_getDevice()} is the current device")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(gpu)  # the handle alone: building a Stream object costs 2 us a call
    if stream.device_index != gpu:
        raise ValueError(f"the tensors are on cuda:{gpu}, the stream on cuda:{stream.device_index}")
    return stream.cuda_stream


def _elsewhere(t: torch.Tensor, gpu: int, name: str) -> None:
    raise ValueError(f"{name} is on cuda:{t.get_device()}, the call's other tensors on cuda:{gpu}")


def _rows(t: torch.Tensor, dtype: torch.dtype, name: str, gpu: Optional[int] = None) -> int:
    """Row stride of a matrix whose rows are contiguous."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise TypeError(f"{name} must be a {dtype} CUDA matrix with contiguous rows")
    if gpu is not None and t.get_device() != gpu:
        _elsewhere(t, gpu, name)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _dense(t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str, gpu: int) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous {dtype} CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.get_device() != gpu:
        _elsewhere(t, gpu, name)
    return t.data_ptr()


def lapsum_route_forward(logits: torch.Tensor, bias: Optional[torch.Tensor], params: RouteParams, idx: torch.Tensor,
                         w: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """idx (int32), w (float32), both tokens x k <- the chosen experts and their weights.  logits: tokens x experts of the
    params' io_dtype with contiguous rows (any row stride); bias: float32, one per expert, or None."""
    stride = _rows(logits, IO_TORCH[params.io_dtype], "logits")
    tokens, experts = logits.shape
    out, gpu = (tokens, params.k), logits.get_device()
    rc = lib().lapsum_route_forward(
        logits.data_ptr(), tokens, experts, stride, None if bias is None else _dense(bias, torch.float32, (experts,), "bias", gpu),
        C.byref(params), _dense(idx, torch.int32, out, "idx", gpu), _dense(w, torch.float32, out, "w", gpu), _stream(stream, gpu))
    if rc:
        _check(rc, "lapsum_route_forward")


def lapsum_route_backward(grad_w: torch.Tensor, logits: torch.Tensor, idx: torch.Tensor, w: torch.Tensor, params: RouteParams,
                          grad_logits: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """grad_logits (tokens x experts, contiguous, the logits' type) <- grad_w (tokens x k, type params.grad_w_dtype)."""
    dtype = IO_TORCH[params.io_dtype]
    stride = _rows(logits, dtype, "logits")
    tokens, experts = logits.shape
    ch, gpu = (tokens, params.k), logits.get_device()
    rc = lib().lapsum_route_backward(
        _dense(grad_w, IO_TORCH[params.grad_w_dtype], ch, "grad_w", gpu), logits.data_ptr(), tokens, experts, stride,
        _dense(idx, torch.int32, ch, "idx", gpu), _dense(w, torch.float32, ch, "w", gpu), C.byref(params),
        _dense(grad_logits, dtype, (tokens, experts), "grad_logits", gpu), _stream(stream, gpu))
    if rc:
        _check(rc, "lapsum_route_backward")


def dispatch_tile_rows(tokens: int, k: int, experts: int, training: bool = False) -> int:
    """Rows per tile that the experts' products are fastest with for this shape."""
    out = C.c_int32()
    _check(lib().lapsum_dispatch_tile_rows(tokens, k, experts, int(training), C.byref(out)), "lapsum_dispatch_tile_rows")
    return out.value


def lapsum_dispatch_describe(tokens: int, k: int, experts: int, tile_rows: int) -> DispatchLayout:
    out = DispatchLayout()
    _check(lib().lapsum_dispatch_describe(tokens, k, experts, tile_rows, C.byref(out)), "lapsum_dispatch_describe")
    return out


def _buffer(n: int, device: torch.device) -> torch.Tensor:
    """n bytes at a multiple of 256"""
    raw = torch.empty(n + 256, dtype=torch.uint8, device=device)
    at = -raw.data_ptr() % 256
    return raw[at:at + n]


def _cuda(device) -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("the LapSum library needs a CUDA device; there is no CPU path")
    return torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())


class _Memory:
    """A buffer of the library's and the streams that use it."""

    def _allocate(self, n: int, device: torch.device) -> None:
        self.buf = _buffer(n, device)
        self.ptr, self.device, self.gpu = self.buf.data_ptr(), self.buf.device, self.buf.get_device()
        self._streams = {torch._C._cuda_getCurrentRawStream(self.gpu)}  # the allocator's memory belongs to the stream that is current

    def _use(self, stream: Optional[torch.cuda.Stream]) -> int:
        """The handle of a call's stream; when the buffer is freed, its memory waits for every stream that was seen here."""
        handle = _stream(stream, self.gpu)
        if handle not in self._streams:
            self.buf.record_stream(stream if stream is not None else torch.cuda.current_stream(self.device))
            self._streams.add(handle)
        return handle


class Dispatch(_Memory):
    """The tables of one batch (lapsum_dispatch_describe): counts, offsets, slot_of (tokens x k), entry_of, tile_expert are
    int32 views of one buffer that lapsum_dispatch fills."""

    def __init__(self, tokens: int, k: int, experts: int, tile_rows: Optional[int] = None, training: bool = False,
                 device: Optional[torch.device] = None):
        dev = _cuda(device)
        self.tokens, self.k, self.experts = int(tokens), int(k), int(experts)
        self.tile_rows = int(tile_rows) if tile_rows is not None else dispatch_tile_rows(tokens, k, experts, training)
        self.layout = L = lapsum_dispatch_describe(self.tokens, self.k, self.experts, self.tile_rows)
        self.capacity, self.bytes = L.capacity, L.bytes
        self._allocate(L.bytes, dev)

        def words(off, n):
            return self.buf[off:off + 4 * n].view(torch.int32)

        self.counts = words(L.off_counts, self.experts)
        self.offsets = words(L.off_offsets, self.experts + 1)
        self.slot_of = words(L.off_slot_of, self.tokens * self.k).view(self.tokens, self.k)
        self.entry_of = words(L.off_entry_of, L.capacity)
        self.tile_expert = words(L.off_tile_expert, L.tiles)


def lapsum_dispatch(idx: torch.Tensor, dispatch: Dispatch, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Fill the tables from idx (int32, tokens x k; entries outside [0, experts) are dropped)."""
    d = dispatch
    rc = lib().lapsum_dispatch(_dense(idx, torch.int32, (d.tokens, d.k), "idx", d.gpu), d.tokens, d.k, d.experts, d.tile_rows, d.ptr,
                               d.bytes, d._use(stream))
    if rc:
        _check(rc, "lapsum_dispatch")


class ExpertsWorkspace(_Memory):
    """Scratch of the experts' products for one shape (lapsum_experts_describe); new_saved() makes the buffer that a
    training forward leaves its activations in, one per forward whose backward is still to come."""

    def __init__(self, dispatch: Dispatch, d: int, f: int, io_dtype: int = IO_BF16, training: bool = False,
                 stream: Optional[torch.cuda.Stream] = None):
        _cuda(dispatch.device)
        p = dispatch
        self.dims = ExpertsDims(p.tokens, p.experts, int(d), int(f), p.k, p.tile_rows, int(io_dtype), int(bool(training)))
        self.training, self.dtype = bool(training), IO_TORCH.get(int(io_dtype))
        out = ExpertsLayout()
        _check(lib().lapsum_experts_describe(C.byref(self.dims), C.byref(out)), "lapsum_experts_describe")
        self.bytes, self.saved_bytes = out.workspace_bytes, out.saved_bytes
        self.shape = (p.tokens, p.k, p.experts, p.tile_rows)
        _stream(stream, p.gpu)  # the checks
        # on the stream that clears it: memory asked for on another one may still be written by what is queued there
        with torch.cuda.stream(stream) if stream is not None else nullcontext():
            self._allocate(self.bytes, p.device)
        _check(lib().lapsum_experts_workspace_init(self.ptr, self.bytes, C.byref(self.dims), self._use(stream)),
               "lapsum_experts_workspace_init")
        self._x = (p.tokens, int(d))
        self._gate_up, self._down = (p.experts, 2 * int(f), int(d)), (p.experts, int(d), int(f))
        self._w = (p.tokens, p.k)
        self._grad_w = {self.dtype: self.dims}  # the dims by grad_w's type
        if self.training:
            self._grad_w[torch.float32] = wide = ExpertsDims.from_buffer_copy(self.dims)
            wide.grad_w_f32 = 1

    def new_saved(self) -> torch.Tensor:
        if not self.training:
            raise ValueError("saved activations belong to a training workspace")
        return _buffer(self.saved_bytes, self.device)

    def status(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        """Status bits (ST_EXPERTS_TIMEOUT); synchronises the stream."""
        out = C.c_uint32()
        _check(lib().lapsum_experts_status(self.ptr, self._use(stream), C.byref(out)), "lapsum_experts_status")
        return out.value


def _same_shape(dispatch: Dispatch, ws: ExpertsWorkspace) -> None:
    if (dispatch.tokens, dispatch.k, dispatch.experts, dispatch.tile_rows) != ws.shape:
        raise ValueError("the dispatch tables and the workspace were made for different shapes")
    if dispatch.gpu != ws.gpu:
        raise ValueError(f"the dispatch tables are on cuda:{dispatch.gpu}, the workspace on cuda:{ws.gpu}")


def _saved(saved: Optional[torch.Tensor], ws: ExpertsWorkspace) -> int:
    if saved is None or not (saved.is_cuda and saved.dtype == torch.uint8 and saved.is_contiguous()):
        raise TypeError("saved must be a buffer of ExpertsWorkspace.new_saved()")
    if saved.get_device() != ws.gpu:
        _elsewhere(saved, ws.gpu, "saved")
    return saved.data_ptr()


def lapsum_experts_forward(x: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor, w: torch.Tensor, dispatch: Dispatch,
                           y: torch.Tensor, ws: ExpertsWorkspace, saved: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
    """y (tokens x d) <- the weighted sum of every token's experts.  x: tokens x d with contiguous rows; w_gate_up: experts x
    2f x d; w_down: experts x d x f; w: tokens x k float32.  `saved` for a training workspace only."""
    _same_shape(dispatch, ws)
    gpu = ws.gpu
    stride = _rows(x, ws.dtype, "x", gpu)
    if x.shape != ws._x:
        raise ValueError(f"x must have shape {ws._x}")
    dispatch._use(stream)
    rc = lib().lapsum_experts_forward(
        x.data_ptr(), stride, _dense(w_gate_up, ws.dtype, ws._gate_up, "w_gate_up", gpu), _dense(w_down, ws.dtype, ws._down, "w_down", gpu),
        _dense(w, torch.float32, ws._w, "w", gpu), dispatch.ptr, dispatch.bytes, None if saved is None else _saved(saved, ws),
        0 if saved is None else saved.numel(), _dense(y, ws.dtype, ws._x, "y", gpu), C.byref(ws.dims), ws.ptr, ws.bytes,
        ws._use(stream))
    if rc:
        _check(rc, "lapsum_experts_forward")


def lapsum_experts_backward(grad_y: torch.Tensor, x: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor, w: torch.Tensor,
                            dispatch: Dispatch, saved: torch.Tensor, grad_x: torch.Tensor, grad_w_gate_up: torch.Tensor,
                            grad_w_down: torch.Tensor, grad_w: torch.Tensor, ws: ExpertsWorkspace,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """Every gradient of lapsum_experts_forward; grad_w has the workspace's 16-bit type or, like w, float32."""
    _same_shape(dispatch, ws)
    gpu = ws.gpu
    gy_stride, x_stride = _rows(grad_y, ws.dtype, "grad_y", gpu), _rows(x, ws.dtype, "x", gpu)
    if x.shape != ws._x or grad_y.shape != ws._x:
        raise ValueError(f"x and grad_y must have shape {ws._x}")
    dims = ws._grad_w.get(grad_w.dtype)
    if dims is None:
        raise TypeError(f"grad_w must be {ws.dtype} or torch.float32")
    dispatch._use(stream)
    rc = lib().lapsum_experts_backward(
        grad_y.data_ptr(), gy_stride, x.data_ptr(), x_stride, _dense(w_gate_up, ws.dtype, ws._gate_up, "w_gate_up", gpu),
        _dense(w_down, ws.dtype, ws._down, "w_down", gpu), _dense(w, torch.float32, ws._w, "w", gpu), dispatch.ptr, dispatch.bytes,
        _saved(saved, ws), saved.numel(), _dense(grad_x, ws.dtype, ws._x, "grad_x", gpu),
        _dense(grad_w_gate_up, ws.dtype, ws._gate_up, "grad_w_gate_up", gpu), _dense(grad_w_down, ws.dtype, ws._down, "grad_w_down", gpu),
        _dense(grad_w, grad_w.dtype, ws._w, "grad_w", gpu), C.byref(dims), ws.ptr, ws.bytes, ws._use(stream))
    if rc:
        _check(rc, "lapsum_experts_backward")
