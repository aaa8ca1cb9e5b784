"""What the dense operators ask for and accept, without a GPU: room for what a call can use, sizes whose results are exact and whose grids exist."""
import ctypes as C

import pytest

import paper_2608_06912_b200 as L
from paper_2608_06912_b200 import binding as B

FAKE = 4096  # 256-byte aligned, never dereferenced: the checks return first
F32, F16, BF16 = L.IO_F32, L.IO_F16, L.IO_BF16


def linear_bytes(rows, n, k, act=L.ACT_NONE, io=BF16, out=BF16):
    layout = B.LinearLayout()
    dims = B.LinearDims(rows, n, k, act, io, out, io, io, F32, 1)
    assert L.lib().lapsum_linear_describe(C.byref(dims), C.byref(layout)) == 0
    return layout.workspace_bytes


@pytest.mark.parametrize("io", [BF16, F16])
def test_a_copied_gradient_has_no_remainder(io):
    """a 16-bit grad_y without an activation is dP: its remainder is zero, so neither room nor a product is spent on it"""
    rows, n, k = 4096, 1000, 64
    plain, one = linear_bytes(rows, n, k, io=io, out=io), rows * n * 2
    assert one <= linear_bytes(rows, n, k, io=io, out=F32) - plain <= one + 4 * (rows + n) + 512
    assert linear_bytes(rows, n, k, io=io, out=io, act=L.ACT_SILU) == linear_bytes(rows, n, k, io=io, out=F32)
    assert plain < 2 * one + 64 * n * 4 * 2 + 148 * 128 * 128 * 4


def test_rows_whose_weights_would_be_too_coarse_are_refused():
    """the sampler's integer weights lose a bit for each doubling of the vocabulary, and their sums two; beyond 2^21 tokens that would show"""
    def call(vocab):
        return L.lib().lapsum_sample(FAKE, 1, vocab, vocab, FAKE, C.byref(L.sample_params()), None, None, None, None, FAKE, None, None, None)

    assert call((1 << 21) + 1) == call(1 << 24) == call(1 << 30) == -2


def test_a_forward_beyond_the_largest_grid_is_refused():
    """2^30 ids with rows of 16 warps each are 2^31 blocks of eight warps, one more than a grid has"""
    rc = L.lib().lapsum_embed_forward(FAKE, 4, 1 << 30, FAKE, 8192, 9, 8192, 1.0, BF16, FAKE, 8192, None)
    assert rc == -2


def test_a_sort_that_would_hold_the_gpu_for_minutes_is_refused():
    """every 512 rows of the table cost a pass over the ids: 2^30 ids into 2^30 rows would be 2^51 reads"""
    def size(tokens, vocab):
        return L.lib().lapsum_embed_workspace_bytes(tokens, vocab, 8, C.byref(C.c_size_t()))

    def back(tokens, vocab):
        return L.lib().lapsum_embed_backward(FAKE, 8, FAKE, 4, tokens, vocab, 8, 1.0, -1, F32, F32, FAKE, FAKE, 1 << 60, None)

    for tokens, vocab in ((1 << 30, 1 << 30), (1 << 23, (1 << 24) + 1), (1 << 30, (1 << 17) + 1)):
        assert size(tokens, vocab) == back(tokens, vocab) == -2
    for tokens, vocab in ((1 << 22, 1 << 24), (1 << 23, 1 << 24), (1 << 30, 1 << 17), (1, 1 << 30), (0, 1 << 30)):
        assert size(tokens, vocab) == 0
