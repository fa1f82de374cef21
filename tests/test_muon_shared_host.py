"""CPU-only: a gradient that shares a value with what a Muon step writes is refused.  The step reads a gradient twice, for the momentum
and for the matrix that is orthogonalised, and has written the momenta in between."""
import ctypes

import pytest

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops


def create(grads, **more):
    """Two bf16 matrices of 8 x 10: weights of 160 bytes, momenta and masters of 320."""
    first = dict(param=4096, m=8192, master=16384)
    second = dict(param=1 << 16, m=1 << 17, master=1 << 18)
    table = (ops._MuonTensor * 2)(*(ops._MuonTensor(**{**dict(rows=8, cols=10, param_type=ops.BF16, grad_type=ops.BF16, module=-1, scale=1.0), **t, **more})
                                    for t in (first, second)))
    h = ctypes.c_void_p()
    return ops.lib().egeria_muon_create(ctypes.byref(h), 2, table, (ctypes.c_void_p * 2)(*grads), 5, 1024, 1 << 24)


@pytest.mark.parametrize("grad", [8192, 8192 - 158, 8192 + 318, 4096, 4096 + 158, 16384, 16384 + 100, 1 << 17, (1 << 16) - 2, (1 << 18) + 318])
@pytest.mark.parametrize("which", [0, 1])
def test_refuses_a_gradient_in_what_is_written(grad, which):
    grads = [1 << 20, 1 << 21]
    grads[which] = grad
    assert create(grads) == eg.ERR_INVALID_ARG


@pytest.mark.parametrize("grads", [(1 << 20, 1 << 20), (8192 - 160, 8192 + 320), (4096 + 160, 4096 - 160), (16384 + 320, 64)])
def test_takes_gradients_beside_it_and_shared_ones(grads):
    """(What is not refused goes on to the device, which is not here, and has no such addresses elsewhere.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    assert create(grads) not in (eg.ERR_INVALID_ARG, eg.OK)


def test_a_float_gradient_is_as_long_as_it_is():
    assert create([8192 - 318, 1 << 21], grad_type=ops.F32) == eg.ERR_INVALID_ARG
    assert create([8192 - 316, 1 << 21], grad_type=ops.F32) == eg.ERR_INVALID_ARG
