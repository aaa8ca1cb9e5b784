"""Sizes and give-up paths of the experts' products that need many slots or many blocks (bounds: tests/experts_util.py)."""
import ctypes as C

import pytest
import torch

import paper_2608_06912_b200 as L
from tests.experts_util import experts_reference
from tests.test_gpu_experts import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("T", [8, 700])
def test_waits_that_run_out_on_every_row_tile(rows, T):
    """A producer that brings nothing and a bound of a millisecond: all roles of a block, and of a pair of blocks, give up and return"""
    r = Run(T, 12, 2, 72, 520, tile_rows=rows, seed=rows)
    L.lapsum_dispatch(r.idx, r.disp)
    rc = L.lib().lapsum_debug_experts_timeout(1000, r.ws.ptr, r.ws.bytes, r.disp.ptr, r.disp.bytes, r.x.contiguous().data_ptr(), r.a.data_ptr(),
                                              r.w.data_ptr(), C.byref(r.ws.dims), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert r.ws.status() == L.ST_EXPERTS_TIMEOUT
    r.ws = L.ExpertsWorkspace(r.disp, 72, 520)
    r.check()  # the context and the tables serve the next call


def test_backward_offsets_beyond_32_bits():
    """1.12 million slots of 2048 columns: more than 2^31 elements per slot buffer, every gradient checked"""
    T, E, k, d, f = 140_000, 16, 8, 2048, 64
    r = Run(T, E, k, d, f, seed=15, tile_rows=128, training=True)
    assert r.disp.capacity * d > 2 ** 31
    out = r()
    torch.cuda.synchronize()
    assert r.ws.status() == 0
    ref = experts_reference(r.x, r.a, r.b, r.idx, r.w, r.gy)
    for name, (want, bound) in ref.items():
        for rows in range(0, want.shape[0], 20_000):
            part = slice(rows, rows + 20_000)
            assert ((out[name][part].double() - want[part]).abs() <= bound[part]).all(), name


@pytest.mark.parametrize("T", [1, 2, 3, 4])
def test_few_tokens_that_share_their_experts(T):
    Run(T, 8, 8, 264, 520, seed=T).check()
    Run(T, 1, 1, 264, 520, torch.float16, seed=T).check()
