"""Host side of the dense entry points (linear, sample, embed): sizes and argument checks, without a GPU."""
import ctypes as C

import pytest

import paper_2608_06912_b200 as L
from paper_2608_06912_b200 import binding as B

FAKE = 4096  # 256-byte aligned, never dereferenced: the checks return first
F32, F16, BF16 = L.IO_F32, L.IO_F16, L.IO_BF16


def linear_dims(**kw):
    base = dict(rows=40, n=72, k=64, activation=L.ACT_NONE, io_dtype=BF16, out_dtype=BF16, bias_dtype=BF16, grad_w_dtype=BF16, pre_dtype=F32, training=0)
    return B.LinearDims(**{**base, **kw})


def describe(**kw):
    out = B.LinearLayout()
    return L.lib().lapsum_linear_describe(C.byref(linear_dims(**kw)), C.byref(out)), out


def test_linear_sizes():
    rc, serve = describe()
    rc2, train = describe(training=1)
    rc3, act = describe(training=1, activation=L.ACT_SILU, n=71)
    rc4, half = describe(training=1, activation=L.ACT_SILU, n=71, pre_dtype=BF16)
    assert rc == rc2 == rc3 == rc4 == 0
    assert serve.pre_bytes == train.pre_bytes == 0 and train.workspace_bytes > serve.workspace_bytes
    assert act.pre_stride == 72 and act.pre_bytes == 40 * 72 * 4 and half.pre_bytes == 40 * 72 * 2
    for n in (1, 8, 200):  # a workspace for some rows serves fewer
        sizes = [describe(rows=r, n=n, training=1)[1].workspace_bytes for r in range(0, 9000, 7)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), -2), (dict(rows=(1 << 30) + 1), -2), (dict(n=0), -2), (dict(n=(1 << 23) + 1), -2), (dict(k=0), -2), (dict(k=60), -2),
    (dict(k=(1 << 20) + 8), -2), (dict(io_dtype=F32), -8), (dict(out_dtype=F16), -8), (dict(bias_dtype=F16), -8), (dict(grad_w_dtype=F16), -8),
    (dict(pre_dtype=F16), -8), (dict(activation=5), -7), (dict(activation=-1), -7), (dict(training=2), -7)])
def test_linear_refuses(bad, code):
    assert describe(**bad)[0] == code


def test_linear_call_checks():
    lib, launches = L.lib(), L.lib().lapsum_launch_count()
    assert lib.lapsum_linear_describe(None, C.byref(B.LinearLayout())) == -1 and lib.lapsum_linear_describe(C.byref(linear_dims()), None) == -1
    need = describe()[1].workspace_bytes

    def fwd(d=None, x=FAKE, xs=64, w=FAKE, bias=None, res=None, rs=72, y=FAKE, ys=72, pre=None, pre_bytes=0, ws=FAKE, n=need):
        return lib.lapsum_linear_forward(x, xs, w, bias, res, rs, y, ys, pre, pre_bytes, C.byref(d or linear_dims()), ws, n, None)

    for name in ("x", "w", "y", "ws"):
        assert fwd(**{name: None}) == -1, name
    assert fwd(x=FAKE + 8) == -9 and fwd(w=FAKE + 8) == -9
    assert fwd(xs=63) == -2 and fwd(xs=68) == -2 and fwd(ys=71) == -2 and fwd(res=FAKE, rs=71) == -2
    assert fwd(ws=FAKE + 16) == -5 and fwd(n=need - 1) == -5
    assert fwd(pre=FAKE) == -7                        # nothing is kept without an activation or without training
    t = linear_dims(training=1, activation=L.ACT_GELU)
    lay = describe(training=1, activation=L.ACT_GELU)[1]
    assert fwd(d=t, n=lay.workspace_bytes) == -1      # training with an activation keeps it
    assert fwd(d=t, n=lay.workspace_bytes, pre=FAKE, pre_bytes=lay.pre_bytes - 1) == -5
    assert fwd(d=linear_dims(rows=0), x=None, w=None, y=None) == 0

    def back(d=t, gy=FAKE, gs=72, x=FAKE, xs=64, w=FAKE, pre=FAKE, pre_bytes=lay.pre_bytes, gx=FAKE, gxs=64, ws=FAKE, n=lay.workspace_bytes):
        return lib.lapsum_linear_backward(gy, gs, x, xs, w, pre, pre_bytes, gx, gxs, FAKE, FAKE, C.byref(d), ws, n, None)

    assert back(d=linear_dims()) == -8                # not a training workspace
    for name in ("gy", "x", "w", "pre", "ws"):
        assert back(**{name: None}) == -1, name
    assert back(gs=71) == -2 and back(xs=60) == -2 and back(gxs=63) == -2 and back(x=FAKE + 8) == -9 and back(pre_bytes=8) == -5
    hook = lib.lapsum_debug_linear_timeout
    assert hook(0, FAKE, FAKE, FAKE, C.byref(linear_dims()), FAKE, need, None) == -7
    assert hook(10, FAKE, FAKE, FAKE, C.byref(linear_dims(rows=4)), FAKE, need, None) == -8
    assert lib.lapsum_launch_count() == launches      # every check came before any device work


def test_sample_defaults_and_checks():
    p = L.sample_params()
    assert (p.temperature, p.top_p, p.min_p, p.top_k, p.io_dtype) == (1.0, 1.0, 0.0, 0, F32)
    with pytest.raises(AttributeError):
        L.sample_params(topk=3)
    lib, launches = L.lib(), L.lib().lapsum_launch_count()

    def call(rows=4, vocab=16, stride=16, logits=FAKE, u=FAKE, token=FAKE, t=None, p_=None, m=None, **kw):
        return lib.lapsum_sample(logits, rows, vocab, stride, u, C.byref(L.sample_params(**kw)), t, None, p_, m, token, None, None, None)

    assert call(rows=0, logits=None) == 0
    assert call(logits=None) == -1 and call(u=None) == -1 and call(token=None) == -1
    assert lib.lapsum_sample(FAKE, 4, 16, 16, FAKE, None, None, None, None, None, FAKE, None, None, None) == -1
    assert call(rows=-1) == -2 and call(vocab=0) == -2 and call(stride=15) == -2 and call(vocab=(1 << 30) + 1, stride=1 << 31) == -2
    nan, inf = float("nan"), float("inf")
    for bad in (dict(temperature=-1.0), dict(temperature=nan), dict(temperature=inf), dict(top_p=0.0), dict(top_p=nan), dict(min_p=-0.1),
                dict(min_p=1.1), dict(min_p=nan), dict(io_dtype=3)):
        assert call(**bad) == -7, bad
    assert lib.lapsum_launch_count() == launches


def test_embed_checks():
    lib, launches = L.lib(), L.lib().lapsum_launch_count()

    def fwd(ids=FAKE, size=4, n=5, table=FAKE, ts=24, vocab=9, d=24, scale=1.0, io=BF16, out=FAKE, os_=24):
        return lib.lapsum_embed_forward(ids, size, n, table, ts, vocab, d, scale, io, out, os_, None)

    assert fwd(n=0, ids=None) == 0
    assert fwd(ids=None) == -1 and fwd(table=None) == -1 and fwd(out=None) == -1
    assert fwd(n=-1) == -2 and fwd(vocab=0) == -2 and fwd(d=0) == -2 and fwd(ts=23) == -2 and fwd(os_=23) == -2
    assert fwd(size=2) == -7 and fwd(scale=float("nan")) == -7 and fwd(scale=1e60) == -7 and fwd(io=3) == -8
    need = C.c_size_t()
    assert lib.lapsum_embed_workspace_bytes(5, 9, 24, C.byref(need)) == 0 and lib.lapsum_embed_workspace_bytes(5, 9, 24, None) == -1
    assert lib.lapsum_embed_workspace_bytes(5, 0, 24, C.byref(C.c_size_t())) == -2

    def back(g=FAKE, gs=24, ids=FAKE, n=5, vocab=9, d=24, io=BF16, gt=F32, grad=FAKE, ws=FAKE, bytes_=need.value):
        return lib.lapsum_embed_backward(g, gs, ids, 4, n, vocab, d, 1.0, -1, io, gt, grad, ws, bytes_, None)

    for name in ("g", "ids", "grad", "ws"):
        assert back(**{name: None}) == -1, name
    assert back(gs=23) == -2 and back(gt=F16) == -8 and back(io=F32, gt=BF16) == -8 and back(ws=FAKE + 16) == -5 and back(bytes_=need.value - 1) == -5
    assert lib.lapsum_launch_count() == launches


def test_workspaces_need_a_gpu():
    import torch

    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        L.LinearWorkspace(4, 8, 8)
    with pytest.raises(RuntimeError):
        L.EmbedWorkspace(4, 8, 8)
