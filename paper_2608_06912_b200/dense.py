"""Binding of the dense entry points of include/lapsum.h, the steps on both sides of the experts: embed, linear, sample.

    embed     lapsum_embed_forward, EmbedWorkspace, lapsum_embed_backward       token ids -> rows of a table; the table's gradient
    linear    LinearWorkspace, lapsum_linear_forward / lapsum_linear_backward   act(x W^T + bias) + residual; its gradients
    sample    lapsum_sample                                                     logits -> the next token of every row

Argument marshalling only, with the rules of experts.py: outputs are the caller's tensors, a call's tensors and its stream are on the
current device, buffers that a workspace owns are recorded on the stream of every call.
"""
from __future__ import annotations

import ctypes as C
from contextlib import nullcontext
from typing import Optional

import torch

from .binding import IO_BF16, IO_F32, IO_TORCH, LinearDims, LinearLayout, SampleParams, _check, lib
from .experts import IO_OF, _cuda, _dense, _elsewhere, _Memory, _rows, _stream

ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2, 3, 4
ACTIVATIONS = {"none": ACT_NONE, "relu": ACT_RELU, "silu": ACT_SILU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH}


# A call's checks are most of a small call's time (a dense layer of one row takes 3 us on the GPU), so what is right is found so by one condition; _dense
# and _rows name what is wrong.
def _flat(t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str, gpu: int) -> int:
    """The address of a contiguous tensor."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == gpu and t.is_contiguous():
        return t.data_ptr()
    return _dense(t, dtype, shape, name, gpu)


def _matrix(t: torch.Tensor, dtype: torch.dtype, shape: tuple, name: str, gpu: int) -> int:
    """The row stride of a matrix of this shape with contiguous rows."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == gpu and t.is_contiguous():
        return shape[1]
    stride = _rows(t, dtype, name, gpu)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return stride


# ------------------------------------------------------------------------------------------------------------ linear
class LinearWorkspace(_Memory):
    """Scratch of act(x W^T + bias) + residual for up to `rows` rows (lapsum_linear_describe).  new_pre() makes the buffer that a training
    forward keeps its pre-activation in (pre_dtype: fp32, or the 16-bit type for half the memory and fewer digits of the slope), one per forward
    whose backward is still to come; without an activation there is none."""

    def __init__(self, rows: int, n: int, k: int, activation: int = ACT_NONE, io_dtype: int = IO_BF16, out_dtype: Optional[int] = None,
                 training: bool = False, pre_dtype: int = IO_F32, device=None, stream: Optional[torch.cuda.Stream] = None):
        dev = _cuda(device)
        out_dtype = io_dtype if out_dtype is None else out_dtype
        self.dims = LinearDims(int(rows), int(n), int(k), int(activation), int(io_dtype), int(out_dtype), int(io_dtype), int(io_dtype),
                               int(pre_dtype), int(bool(training)))
        out = LinearLayout()
        _check(lib().lapsum_linear_describe(C.byref(self.dims), C.byref(out)), "lapsum_linear_describe")
        self.rows, self.n, self.k, self.training = int(rows), int(n), int(k), bool(training)
        self.dtype, self.out_dtype, self.pre_dtype = IO_TORCH[io_dtype], IO_TORCH[out_dtype], IO_TORCH[pre_dtype]
        self._dims, self._w, self._b = {}, (self.n, self.k), (self.n,)  # _dims: a call's dims by its rows and types
        self.bytes, self.pre_bytes, self.pre_stride = out.workspace_bytes, out.pre_bytes, out.pre_stride
        with torch.cuda.device(dev), torch.cuda.stream(stream) if stream is not None else nullcontext():
            self._allocate(self.bytes, dev)
            _check(lib().lapsum_linear_workspace_init(self.ptr, self.bytes, C.byref(self.dims), self._use(stream)), "lapsum_linear_workspace_init")

    def new_pre(self) -> Optional[torch.Tensor]:
        """rows x n in memory of rows that are whole 16-byte vectors; None without an activation"""
        if not self.training:
            raise ValueError("a kept pre-activation belongs to a training workspace")
        if not self.pre_bytes:
            return None
        return torch.empty(self.rows, self.pre_stride, dtype=self.pre_dtype, device=self.device)[:, :self.n]

    def status(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        """Status bits (ST_LINEAR_TIMEOUT); synchronises the stream."""
        out = C.c_uint32()
        _check(lib().lapsum_linear_status(self.ptr, self._use(stream), C.byref(out)), "lapsum_linear_status")
        return out.value

    def _call(self, x: torch.Tensor, wide_bias: bool, wide_grad: bool = False) -> tuple:
        """(reference to this call's dims, rows, x's row stride)"""
        shape = x.shape
        rows = shape[0] if len(shape) == 2 else -1
        dims = self._dims.get((rows, wide_bias, wide_grad))
        if dims is None or shape[1] != self.k:
            _rows(x, self.dtype, "x", self.gpu)
            if shape[1] != self.k or rows > self.rows:
                raise ValueError(f"x must have up to {self.rows} rows of {self.k}, not shape {tuple(shape)}")
            made = LinearDims.from_buffer_copy(self.dims)
            made.rows, made.bias_dtype, made.grad_w_dtype = rows, IO_F32 if wide_bias else made.bias_dtype, IO_F32 if wide_grad else made.grad_w_dtype
            if len(self._dims) >= 256:
                self._dims.clear()
            dims = self._dims[rows, wide_bias, wide_grad] = C.byref(made)
        return dims, rows, _matrix(x, self.dtype, (rows, self.k), "x", self.gpu)

    def _kept(self, pre: Optional[torch.Tensor], rows: int) -> tuple:
        if not self.pre_bytes:
            if pre is not None:
                raise ValueError("pre belongs to a training workspace with an activation")
            return None, 0
        if pre is None:
            raise TypeError("pre must be a buffer of LinearWorkspace.new_pre()")
        stride = _rows(pre, self.pre_dtype, "pre", self.gpu)
        if pre.shape[1] != self.n or pre.shape[0] < rows or (stride != self.pre_stride and pre.shape[0] > 1):
            raise ValueError("pre must be a buffer of LinearWorkspace.new_pre()")
        room = pre.untyped_storage().nbytes() - pre.storage_offset() * pre.element_size()
        return pre.data_ptr(), room


def lapsum_linear_forward(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor], residual: Optional[torch.Tensor], y: torch.Tensor,
                          ws: LinearWorkspace, pre: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """y (rows x n, the workspace's out_dtype) <- act(x w^T + bias) + residual.  x: rows x k with contiguous rows; w: n x k; bias: n, the
    workspace's 16-bit type or float32; residual like y (or y itself)."""
    gpu, kind = ws.gpu, ws.out_dtype
    wide = bias is not None and bias.dtype is torch.float32
    dims, rows, stride = ws._call(x, wide)
    out = (rows, ws.n)
    at, room = ws._kept(pre, rows) if pre is not None or ws.pre_bytes else (None, 0)
    rc = lib().lapsum_linear_forward(
        x.data_ptr(), stride, _flat(w, ws.dtype, ws._w, "w", gpu), None if bias is None else _flat(bias, torch.float32 if wide else ws.dtype, ws._b, "bias", gpu),
        None if residual is None else residual.data_ptr(), 0 if residual is None else _matrix(residual, kind, out, "residual", gpu), y.data_ptr(),
        _matrix(y, kind, out, "y", gpu), at, room, dims, ws.ptr, ws.bytes, ws._use(stream))
    if rc:
        _check(rc, "lapsum_linear_forward")


def lapsum_linear_backward(grad_y: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor], grad_x: Optional[torch.Tensor],
                           grad_w: Optional[torch.Tensor], grad_bias: Optional[torch.Tensor], ws: LinearWorkspace,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
    """The gradients of lapsum_linear_forward that are not None; grad_w and grad_bias have the workspace's 16-bit type or float32.  The
    residual's gradient is grad_y."""
    gpu = ws.gpu
    wide, wide_w = grad_bias is not None and grad_bias.dtype is torch.float32, grad_w is not None and grad_w.dtype is torch.float32
    dims, rows, stride = ws._call(x, wide, wide_w)
    at, room = ws._kept(pre, rows) if pre is not None or ws.pre_bytes else (None, 0)
    rc = lib().lapsum_linear_backward(
        grad_y.data_ptr(), _matrix(grad_y, ws.out_dtype, (rows, ws.n), "grad_y", gpu), x.data_ptr(), stride, _flat(w, ws.dtype, ws._w, "w", gpu), at, room,
        None if grad_x is None else grad_x.data_ptr(), 0 if grad_x is None else _matrix(grad_x, ws.dtype, (rows, ws.k), "grad_x", gpu),
        None if grad_w is None else _flat(grad_w, torch.float32 if wide_w else ws.dtype, ws._w, "grad_w", gpu),
        None if grad_bias is None else _flat(grad_bias, torch.float32 if wide else ws.dtype, ws._b, "grad_bias", gpu), dims, ws.ptr, ws.bytes,
        ws._use(stream))
    if rc:
        _check(rc, "lapsum_linear_backward")


# ------------------------------------------------------------------------------------------------------------ sample
def sample_params(**overrides) -> SampleParams:
    """lapsum_sample_default_params with the named fields replaced."""
    p = SampleParams()
    lib().lapsum_sample_default_params(C.byref(p))
    for key, val in overrides.items():
        if not hasattr(p, key):
            raise AttributeError(key)
        setattr(p, key, val)
    return p


def lapsum_sample(logits: torch.Tensor, u: torch.Tensor, params: SampleParams, token: torch.Tensor, logprob: Optional[torch.Tensor] = None,
                  kept: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                  top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """token (int32, one per row) <- the next token of every row of logits (rows x vocab of the params' io_dtype, up to 2^21 tokens, contiguous
    rows, any row stride) for the random numbers u (float32, one per row, in [0, 1)).  logprob (float32), kept (int32): see lapsum_sample in the header.
    temperature, top_p, min_p (float32) and top_k (int32), one per row, replace the params' value for all rows."""
    stride = _rows(logits, IO_TORCH[params.io_dtype], "logits")
    rows, vocab = logits.shape
    gpu, f, i, n = logits.get_device(), torch.float32, torch.int32, (rows,)
    rc = lib().lapsum_sample(
        logits.data_ptr(), rows, vocab, stride, _flat(u, f, n, "u", gpu), C.byref(params),
        None if temperature is None else _flat(temperature, f, n, "temperature", gpu), None if top_k is None else _flat(top_k, i, n, "top_k", gpu),
        None if top_p is None else _flat(top_p, f, n, "top_p", gpu), None if min_p is None else _flat(min_p, f, n, "min_p", gpu),
        _flat(token, i, n, "token", gpu), None if logprob is None else _flat(logprob, f, n, "logprob", gpu),
        None if kept is None else _flat(kept, i, n, "kept", gpu), _stream(stream, gpu))
    if rc:
        _check(rc, "lapsum_sample")


# ------------------------------------------------------------------------------------------------------------- embed
_ID_BYTES = {torch.int32: 4, torch.int64: 8}


def _ids(ids: torch.Tensor, gpu: int) -> tuple:
    size, shape = _ID_BYTES.get(ids.dtype), ids.shape
    if size is None or len(shape) != 1 or not ids.is_contiguous() or not ids.is_cuda:
        raise TypeError("ids must be a contiguous int32 or int64 CUDA vector")
    if ids.get_device() != gpu:
        _elsewhere(ids, gpu, "ids")
    return ids.data_ptr(), size, shape[0]


def lapsum_embed_forward(ids: torch.Tensor, table: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
                         stream: Optional[torch.cuda.Stream] = None) -> None:
    """out (tokens x d) <- scale * table[ids]; ids outside the table give zeros.  ids: int32 or int64; table: vocab x d, float32, float16
    or bfloat16, contiguous rows; out like the table."""
    dtype = table.dtype
    io = IO_OF.get(dtype)
    if io is None:
        raise TypeError("table must be float32, float16 or bfloat16")
    stride, gpu = _rows(table, dtype, "table"), table.get_device()
    at, size, tokens = _ids(ids, gpu)
    vocab, d = table.shape
    rc = lib().lapsum_embed_forward(at, size, tokens, table.data_ptr(), stride, vocab, d, scale, io, out.data_ptr(),
                                    _matrix(out, dtype, (tokens, d), "out", gpu), _stream(stream, gpu))
    if rc:
        _check(rc, "lapsum_embed_forward")


class EmbedWorkspace(_Memory):
    """Scratch of the table's gradient for up to `tokens` ids (lapsum_embed_workspace_bytes)."""

    def __init__(self, tokens: int, vocab: int, d: int, device=None):
        dev = _cuda(device)
        out = C.c_size_t()
        _check(lib().lapsum_embed_workspace_bytes(int(tokens), int(vocab), int(d), C.byref(out)), "lapsum_embed_workspace_bytes")
        self.tokens, self.vocab, self.d, self.bytes = int(tokens), int(vocab), int(d), out.value
        self._allocate(self.bytes, dev)


def lapsum_embed_backward(grad_out: torch.Tensor, ids: torch.Tensor, grad_table: torch.Tensor, ws: EmbedWorkspace, scale: float = 1.0,
                          skip: int = -1, stream: Optional[torch.cuda.Stream] = None) -> None:
    """grad_table (vocab x d, written in full; grad_out's type or float32) <- scale times the sums of grad_out's rows by id; `skip` (the padding
    id) and ids outside the table add nothing."""
    if grad_out.dtype not in IO_OF:
        raise TypeError("grad_out must be float32, float16 or bfloat16")
    gpu = ws.gpu
    at, size, tokens = _ids(ids, gpu)
    if tokens > ws.tokens:
        raise ValueError(f"the workspace is for up to {ws.tokens} ids, not {tokens}")
    wide = torch.float32 if grad_table.dtype == torch.float32 else grad_out.dtype
    rc = lib().lapsum_embed_backward(
        grad_out.data_ptr(), _matrix(grad_out, grad_out.dtype, (tokens, ws.d), "grad_out", gpu), at, size, tokens, ws.vocab, ws.d, scale, skip,
        IO_OF[grad_out.dtype], IO_OF[wide], _flat(grad_table, wide, (ws.vocab, ws.d), "grad_table", gpu), ws.ptr, ws.bytes, ws._use(stream))
    if rc:
        _check(rc, "lapsum_embed_backward")
