"""Which calls of a few tokens take the products without the tensor core, counted in launches: two there, three or four on tiles."""
import pytest
import torch

import paper_2608_06912_b200 as L
from tests.test_gpu_experts import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k,d,f,few", [
    (1, 8, 8, 2048, 1024, True), (1, 1, 1, 2048, 1024, True), (4, 64, 2, 1024, 1024, True), (2, 64, 8, 2048, 1024, True),
    (4, 8, 8, 264, 136, True),     # every expert four times, but the weights are small: two launches fewer count for more
    (3, 8, 8, 2048, 1024, False), (4, 8, 8, 2048, 1024, False), (4, 16, 8, 2048, 1024, False), (4, 8, 2, 4096, 1792, False),  # 200 MB and more read again
    (5, 64, 1, 64, 64, False),
])
def test_tokens_that_share_large_experts_take_tiles(T, E, k, d, f, few):
    """Measured, few / tiles: 4 tokens on 8 of 8 experts of 2048 x 1024 62 / 37 us, one token 27 / 36 us, 4 tokens on 2 of 4 experts of
    1000 x 520 15 / 24 us"""
    r = Run(T, E, k, d, f, seed=T + E)
    L.lapsum_dispatch(r.idx, r.disp)
    y = torch.empty_like(r.x)
    before = L.lapsum_launch_count()
    L.lapsum_experts_forward(r.x, r.a, r.b, r.w, r.disp, y, r.ws)
    launches = L.lapsum_launch_count() - before
    assert (launches == 2) == few, launches
    r.check()
