"""The gated block and the Muon step together, as the example uses them: norm, block, gate and residual stream, backward to the first
block that trains, updates under the evaluation's mask."""
import sys
from pathlib import Path

import pytest
import torch

from paper_2201_06227_b200 import ops
from test_ops_gpu import DEV, rand

pytestmark = pytest.mark.gpu
sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
import train_frozen_blocks as example  # noqa: E402


@pytest.mark.parametrize("gated,muon,bits", [(True, True, 32), (True, False, 8), (False, True, 32)])
def test_example_trains_and_leaves_frozen_blocks_alone(gated, muon, bits):
    losses, frozen, model, at_freeze = example.train(blocks=3, hidden=128, batch=32, seq=8, steps=60, every=4, window=3, tolerance=2e-3,
                                                     gated=gated, muon=muon, bits=bits, log=lambda _: None)
    assert all(v == v and v < float("inf") for v in losses)
    assert all(torch.isfinite(v).all() for p in model.params for v in p.values())
    assert len(at_freeze) == frozen
    for i, kept in at_freeze.items():
        for k, v in kept.items():
            assert torch.equal(model.params[i][k], v), (i, k)


def test_gradients_of_gated_blocks():
    """The example's backward pass against autograd on the same model in 64 bits.  Each hand-over between two calls rounds by 2^-8 at most,
    a block has eight of them either way and two blocks follow one another: 2 * 16 * 2^-8 / sqrt(12) = 0.036 in the 2-norm were they all to
    add up; gradients that are wrong are off by their own size."""
    blocks, hidden, rows = 2, 96, 160
    handle = ops.Ops(max(ops.egeria_gated_workspace_bytes(rows, hidden, example.gated_width(hidden), hidden), ops.egeria_norm_workspace_bytes(rows, hidden)), DEV)
    model = example.Blocks(blocks, hidden, handle, 5, DEV, gated=True)
    x, dh = rand(rows, hidden, seed=1), rand(rows, hidden, seed=2)
    _, kept, _ = model.forward(x)
    grads = [{k: torch.zeros_like(v) for k, v in p.items()} for p in model.params]
    model.backward(dh, kept, 0, grads)

    params = [{k: v.double().requires_grad_() for k, v in p.items()} for p in model.params]
    norm = lambda a, w, b: torch.nn.functional.layer_norm(a, (hidden,), w, b, 1e-5)  # noqa: E731
    stream = x.double()
    h = norm(stream, None, None)
    for p in params:
        f = (torch.nn.functional.silu(h @ p["w_gate"].t()) * (h @ p["w_up"].t())) @ p["w_down"].t()
        stream = stream + p["gate"] * norm(f, p["w_post"], p["b_post"])
        h = norm(stream, p["w_pre"], p["b_pre"])
    (h * dh.double()).sum().backward()
    for i, p in enumerate(params):
        for k, v in p.items():
            off = float((grads[i][k].double() - v.grad).norm() / v.grad.norm())
            assert off <= 0.036, (i, k, off)
    handle.check_device_status()
