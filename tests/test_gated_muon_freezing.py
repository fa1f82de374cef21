"""The example's loop with gated blocks and the Muon step, where blocks do freeze: the evaluation's mask stops the matrices of a frozen
block at once and for good, and those behind it go on."""
import sys
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
import train_frozen_blocks as example  # noqa: E402

BLOCKS, HIDDEN, MATRICES = 6, 64, ("w1", "w2", "w_gate", "w_up", "w_down")


@pytest.mark.parametrize("gated,muon,bits", [(True, True, 32), (True, False, 8), (False, True, 32)])
def test_frozen_blocks_stop_and_the_others_go_on(gated, muon, bits):
    """With a tolerance above any slope every evaluation counts towards freezing the front, which takes `window` = 3 of them at least:
    fifteen evaluations freeze one block at least and five of the six at most."""
    lines = []
    losses, frozen, model, at_freeze = example.train(blocks=BLOCKS, hidden=HIDDEN, batch=16, seq=4, steps=60, every=4, window=3, tolerance=1e9,
                                                     gated=gated, muon=muon, bits=bits, log=lines.append)
    assert len(losses) == 60 and all(v == v and v < float("inf") for v in losses)
    assert 1 <= frozen < BLOCKS and sorted(at_freeze) == list(range(frozen)) and lines
    start = example.Blocks(BLOCKS, HIDDEN, None, 1, "cuda", gated)
    for i, p in enumerate(model.params):
        for k, v in p.items():
            assert torch.isfinite(v).all(), (i, k)
            if i in at_freeze:
                assert torch.equal(v, at_freeze[i][k]), (i, k)
        for k in MATRICES:
            if k in p:
                assert not torch.equal(p[k], start.params[i][k]), (i, k)      # every matrix moved while it was free to
    last, first = model.params[-1], at_freeze[0]
    for k in MATRICES:
        if k in last:                                                          # and the last one's by more than the first one's, which stopped
            assert (last[k] - start.params[-1][k]).float().norm() > (first[k] - start.params[0][k]).float().norm(), k
