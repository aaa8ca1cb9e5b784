"""Objects of the mixture-of-experts calls that are dropped while another stream still works with their memory."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.test_gpu_experts import Run

pytestmark = pytest.mark.gpu


def step(r, disp, ws, out, stream=None):
    L.lapsum_dispatch(r.idx, disp, stream)
    L.lapsum_experts_forward(r.x, r.a, r.b, r.w, disp, out["y"], ws, saved=r.saved, stream=stream)
    L.lapsum_experts_backward(r.gy, r.x, r.a, r.b, r.w, disp, r.saved, out["grad_x"], out["grad_w_gate_up"], out["grad_w_down"], out["grad_w"],
                              ws, stream=stream)


@pytest.mark.parametrize("how", ["current", "argument"])
def test_dropped_tables_and_workspace_stay_until_the_stream_is_done(how):
    r = Run(500, 8, 2, 264, 136, training=True, seed=21)
    want = {n: v.clone() for n, v in r().items()}
    out = {n: torch.zeros_like(v) for n, v in want.items()}
    side = torch.cuda.Stream()
    disp = L.Dispatch(500, 2, 8, tile_rows=r.disp.tile_rows)
    ws = L.ExpertsWorkspace(disp, 264, 136, training=True)
    torch.cuda.synchronize()
    sizes = (disp.bytes + 256, ws.bytes + 256)
    held = [(o.buf.untyped_storage().data_ptr(), o.buf.untyped_storage().nbytes()) for o in (disp, ws)]
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # some 60 ms before the first kernel
        if how == "current":
            step(r, disp, ws, out)
    if how == "argument":
        step(r, disp, ws, out, side)
    assert not side.query()
    del disp, ws
    fresh = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes * 3]
    assert not side.query()  # the kernels have not run yet, so the memory must still be theirs
    for t in fresh:
        lo, hi = t.data_ptr(), t.data_ptr() + t.numel()
        assert all(hi <= p or lo >= p + n for p, n in held)
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(out[n], want[n]), n


def test_a_workspace_made_for_another_stream():
    r = Run(64, 4, 2, 64, 72, seed=22)
    want = r()["y"].clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = L.ExpertsWorkspace(r.disp, 64, 72, stream=side)
    y = torch.empty_like(want)
    side.wait_stream(torch.cuda.current_stream())
    L.lapsum_experts_forward(r.x, r.a, r.b, r.w, r.disp, y, ws, stream=side)
    assert ws.status(side) == 0
    assert torch.equal(y, want)
