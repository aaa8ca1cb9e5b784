"""Host side of the mixture-of-experts entry points: sizes and argument checks, without a GPU."""
import ctypes as C

import pytest

import paper_2608_06912_b200 as L
from paper_2608_06912_b200 import binding as B

FAKE = 4096  # 256-byte aligned, never dereferenced: the checks return first


def test_route_defaults_and_checks():
    p = L.route_params()
    assert (p.k, p.score, p.groups, p.groups_kept, p.group_top, p.renormalise, p.scale) == (1, L.ROUTE_SOFTMAX, 1, 1, 2, 1, 1.0)
    with pytest.raises(AttributeError):
        L.route_params(top_k=3)
    lib = L.lib()

    def fwd(tokens=4, experts=16, stride=16, logits=FAKE, idx=FAKE, w=FAKE, **kw):
        return lib.lapsum_route_forward(logits, tokens, experts, stride, None, C.byref(L.route_params(**{"k": 2, **kw})), idx, w, None)

    assert fwd(tokens=0, logits=None) == 0
    assert fwd(logits=None) == -1 and fwd(idx=None) == -1 and fwd(w=None) == -1
    assert lib.lapsum_route_forward(FAKE, 4, 16, 16, None, None, FAKE, FAKE, None) == -1
    assert fwd(tokens=-1) == -2 and fwd(experts=0) == -2 and fwd(experts=1025, stride=1025) == -2 and fwd(stride=15) == -2
    for bad in (dict(k=0), dict(k=33), dict(k=17), dict(groups=3), dict(groups=33), dict(groups=4, groups_kept=5), dict(groups_kept=0),
                dict(group_top=0), dict(group_top=3), dict(scale=0.0), dict(scale=float("inf")), dict(scale=1e-60), dict(score=3),
                dict(io_dtype=3), dict(grad_w_dtype=-1)):
        assert fwd(**bad) == -7, bad
    p = L.route_params(k=2)
    assert lib.lapsum_route_backward(None, FAKE, 4, 16, 16, FAKE, FAKE, C.byref(p), FAKE, None) == -1
    assert lib.lapsum_route_backward(FAKE, FAKE, 4, 16, 16, FAKE, FAKE, C.byref(p), None, None) == -1


@pytest.mark.parametrize("tokens,k,experts,rows,capacity", [
    (0, 2, 8, 16, 0), (1, 8, 128, 16, 128), (1, 1, 1, 128, 128), (32, 8, 128, 16, 2176), (65536, 8, 128, 128, 540544), (3, 2, 4, 64, 256),
])
def test_dispatch_sizes(tokens, k, experts, rows, capacity):
    d = L.lapsum_dispatch_describe(tokens, k, experts, rows)
    assert d.capacity == capacity and d.tiles == capacity // rows
    offs = [d.off_counts, d.off_offsets, d.off_slot_of, d.off_entry_of, d.off_tile_expert, d.off_partial]
    assert all(o % 256 == 0 for o in offs) and offs == sorted(offs) and d.bytes >= 4 * (2 * experts + 1 + tokens * k + capacity)
    # the slots hold every way the entries can fall: `used` experts with one row more than full tiles
    used = min(tokens * k, experts)
    assert capacity >= tokens * k and capacity + rows > tokens * k + used * (rows - 1) >= capacity


def test_row_tiles_by_mean_load():
    t = L.dispatch_tile_rows
    assert t(1, 8, 128) == 16 and t(0, 1, 4) == 16
    assert t(128, 8, 64) == 32 and t(256, 8, 64) == 64 and t(1024, 8, 64) == 128
    assert t(16384, 8, 64) == 256 and t(16384, 8, 64, True) == 256
    assert t(1, 8, 128, True) == 64  # training needs 64 rows or more
    with pytest.raises(L.LapsumError):
        t(1, 0, 4)


def test_dispatch_checks():
    lib = L.lib()
    d = L.lapsum_dispatch_describe(4, 2, 8, 16)
    call = lambda idx=FAKE, T=4, k=2, E=8, rows=16, buf=FAKE, n=d.bytes: lib.lapsum_dispatch(idx, T, k, E, rows, buf, n, None)  # noqa: E731
    assert call(idx=None) == -1 and call(buf=None) == -1 and call(buf=FAKE + 16) == -5 and call(n=d.bytes - 1) == -5
    assert call(rows=24) == -7 and call(k=33) == -2 and call(E=1025) == -2 and call(T=-1) == -2 and call(T=1 << 30) == -2


def test_experts_sizes_and_checks():
    lib = L.lib()
    launches = lib.lapsum_launch_count()

    def dims(**kw):
        base = dict(tokens=40, experts=8, d=64, f=72, k=2, tile_rows=64, io_dtype=L.IO_BF16, training=0)
        return B.ExpertsDims(**{**base, **kw})

    def describe(**kw):
        out = B.ExpertsLayout()
        return lib.lapsum_experts_describe(C.byref(dims(**kw)), C.byref(out)), out

    rc, serve = describe()
    rc2, train = describe(training=1)
    assert rc == rc2 == 0 and serve.saved_bytes == 0 and train.saved_bytes > 0 and train.workspace_bytes > 0
    cap = L.lapsum_dispatch_describe(40, 2, 8, 64).capacity
    assert train.saved_bytes >= cap * 72 * 6 and serve.workspace_bytes >= cap * (64 + 72) * 2
    assert lib.lapsum_experts_describe(None, C.byref(serve)) == -1 and lib.lapsum_experts_describe(C.byref(dims()), None) == -1
    for bad, code in ((dict(d=60), -2), (dict(f=4), -2), (dict(d=0), -2), (dict(io_dtype=L.IO_F32), -8), (dict(tile_rows=48), -7),
                      (dict(training=1, tile_rows=32), -7), (dict(training=2), -7), (dict(k=0), -2), (dict(experts=2000), -2)):
        assert describe(**bad)[0] == code, bad

    disp = L.lapsum_dispatch_describe(40, 2, 8, 64)

    def fwd(d=None, x=FAKE, stride=64, a=FAKE, b=FAKE, w=FAKE, tab=FAKE, tab_bytes=disp.bytes, saved=None, y=FAKE, ws=FAKE,
            ws_bytes=serve.workspace_bytes):
        return lib.lapsum_experts_forward(x, stride, a, b, w, tab, tab_bytes, saved, 0, y, C.byref(d or dims()), ws, ws_bytes, None)

    for name in ("x", "a", "b", "w", "tab", "y", "ws"):
        assert fwd(**{name: None}) == -1, name
    for name in ("x", "a", "b", "y"):
        assert fwd(**{name: FAKE + 8}) == -9, name
    assert fwd(stride=63) == -2 and fwd(stride=68) == -2
    assert fwd(tab=FAKE + 16) == -5 and fwd(tab_bytes=disp.bytes - 1) == -5 and fwd(ws=FAKE + 16) == -5
    assert fwd(ws_bytes=serve.workspace_bytes - 1) == -5
    assert fwd(saved=FAKE) == -7                                   # serving keeps nothing
    t = dims(training=1)
    assert fwd(d=t, ws_bytes=train.workspace_bytes) == -1          # training needs the buffer
    assert fwd(d=t, ws_bytes=train.workspace_bytes, saved=FAKE) == -5  # of zero bytes
    back = lib.lapsum_experts_backward
    assert back(FAKE, 64, FAKE, 64, FAKE, FAKE, FAKE, FAKE, disp.bytes, FAKE, 1 << 40, FAKE, FAKE, FAKE, FAKE, C.byref(dims()), FAKE, 1 << 40,
                None) == -8
    assert back(FAKE, 60, FAKE, 64, FAKE, FAKE, FAKE, FAKE, disp.bytes, FAKE, 1 << 40, FAKE, FAKE, FAKE, FAKE, C.byref(t), FAKE, 1 << 40, None) == -2
    assert lib.lapsum_error_string(-9).decode() == "a tensor does not start at a multiple of 16 bytes"
    assert lib.lapsum_launch_count() == launches  # every check above came before any device work


def test_a_dispatch_needs_a_gpu():
    import torch

    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        L.Dispatch(4, 2, 8)
