"""The example that runs the operators and the freezing rule together as a training loop."""
import sys
from pathlib import Path

import pytest
import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_blocks_train_and_frozen_ones_stay(bits):
    import train_frozen_blocks as example
    losses, frozen, model, at_freeze = example.train(blocks=3, hidden=64, batch=16, seq=4, steps=120, bits=bits, log=lambda *_: None)
    assert all(v == v for v in losses)
    assert sum(losses[-10:]) < 0.8 * sum(losses[:10])           # it learns
    assert frozen >= 1 and sorted(at_freeze) == list(range(frozen))
    for i, then in at_freeze.items():                           # and a frozen block is as it was when it froze
        for k, v in then.items():
            assert torch.equal(v, model.params[i][k]), (i, k)
    assert not torch.equal(model.params[-1]["w1"], example.Blocks(3, 64, None, 1, "cuda").params[-1]["w1"])
