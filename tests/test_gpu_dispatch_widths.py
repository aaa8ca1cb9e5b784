"""Dispatch at every width around those where its kernel's shared memory passes what a launch gets without asking."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch, sys
sys.path.insert(0, {root!r})
import paper_2608_06912_b200 as L
from tests.experts_util import chosen, dispatch_reference
gen = torch.Generator().manual_seed(0)
for E in {widths!r}:
    idx = chosen(90, E, 6, gen, drop=0.1, device="cpu")
    d = L.Dispatch(90, 6, E, tile_rows=16)
    L.lapsum_dispatch(idx.cuda(), d)
    counts, offsets, slot_of, entry_of = dispatch_reference(idx, E, 16)
    assert d.counts.tolist() == counts and d.offsets.tolist() == offsets, E
    assert d.slot_of.reshape(-1).tolist() == slot_of and d.entry_of.tolist()[:len(entry_of)] == entry_of, E
print("ok")
"""


@pytest.mark.parametrize("widths", [[641, 642], [643], [644], [645, 646], [640, 1024, 645], [257, 600]])
def test_dispatch_in_a_fresh_process(widths):
    """in a process of its own: an earlier call with more experts would have asked for the memory already"""
    out = subprocess.run([sys.executable, "-c", CODE.format(root=ROOT, widths=widths)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stderr[-2000:]


def test_widths_taken_in_turn_by_several_threads():
    """every thread's launch has the memory that it needs, whatever widths the others use"""
    import threading

    import torch

    import paper_2608_06912_b200 as L
    from tests.experts_util import dispatch_reference

    failures = []

    def work(widths):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                made = []
                for E in widths * 40:
                    idx = torch.arange(60, dtype=torch.int32).view(20, 3) * 17 % E
                    d = L.Dispatch(20, 3, E, tile_rows=16)
                    L.lapsum_dispatch(idx.cuda(), d)
                    made.append((idx, E, d))
                stream.synchronize()
                for idx, E, d in made:
                    assert d.counts.tolist() == dispatch_reference(idx, E, 16)[0], E
        except Exception as e:  # noqa: BLE001
            failures.append(repr(e))

    threads = [threading.Thread(target=work, args=(w,)) for w in ([660, 1024], [700, 650], [1000, 668], [300, 900])]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failures, failures[:3]
