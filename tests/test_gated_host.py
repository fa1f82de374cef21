"""CPU-only checks of the gated feed-forward blocks: workspace sizes, refusals."""
import random

import pytest
import torch

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops


def test_workspace_sizes():
    size = ops.egeria_gated_workspace_bytes
    assert size(0, 64, 64, 64) >= ops.OPS_WORKSPACE_MIN
    for bad in ((-1, 64, 64, 64), (1, 0, 64, 64), (1, 64, 0, 64), (1, 64, 64, 0), (2 ** 31, 64, 64, 64), (1, 2 ** 31, 64, 64), (1, 64, 2 ** 31, 64), (1, 64, 64, 2 ** 31)):
        assert size(*bad) == 0, bad
    most = 2 ** 31 - 1024                                   # sizes whose products leave 64 bits: more than any workspace has
    assert size(most, most, most, most) >= 2 ** 61 and size(most, 1, most, 1) >= 2 ** 61 and size(1, most, most, 1) >= 2 ** 61
    # copies of every operand and the three hidden matrices of a backward pass
    assert size(1000, 1001, 999, 1003) >= 2 * (1000 * (1008 + 1008) + 999 * 2 * 1008 + 1003 * 1000 + 3 * 1000 * 1008)


def test_workspace_never_falls_as_a_size_grows():
    r = random.Random(6)
    for _ in range(20000):
        big = [int(2 ** r.uniform(0, m)) for m in (17, 13, 14, 13)]
        small = [r.choice((v, max(1, v - 1), r.randint(1, v))) for v in big]
        assert ops.egeria_gated_workspace_bytes(*small) <= ops.egeria_gated_workspace_bytes(*big), (small, big)


def test_refusals_of_the_entry_points():
    L = ops.lib()
    for call in (L.egeria_gated_forward, L.egeria_gated_backward):
        assert call(None, None, bytes(512)) == eg.ERR_INVALID_ARG
        assert call(None, None, None) == eg.ERR_INVALID_ARG


def test_extension_refuses_what_is_no_tensor_or_not_on_the_gpu():
    n = ops._native()
    x = torch.zeros(4, 4, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        n.gated_forward(0, 0, 0, 0, x, x, x, x, None, None, None, 4, None, False)                    # an argument short
    with pytest.raises(ValueError):
        n.gated_forward(0, 0, 0, 0, x, x, 3, x, None, None, None, 4, None, False, None)
    with pytest.raises(ValueError):
        n.gated_forward(0, 0, 0, 0, x, x, x, x, None, None, None, 4, None, False, None)              # host memory
    with pytest.raises(ValueError):
        n.gated_backward(0, 0, 0, 0, x, x, x, x, x, x, x, 4, True, True, False)
    with pytest.raises(ValueError):
        n.gated_backward(0, 0, 0, 0, x, None, x, x, x, x, x, 4, True, True, False)                   # no x for the weights' gradients
