"""CPU-only checks of the Muon step's C ABI: layout, workspace sizes, refusals."""
import ctypes
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops

HEADER = Path(__file__).resolve().parent.parent / "include" / "egeria_ops.h"


def test_struct_has_the_headers_layout(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    m = ops._MuonTensor
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include "egeria_ops.h"\n#include <stdio.h>\nint main(void) {\n    printf("size %zu\\n", sizeof(egeria_muon_tensor));\n' +
                   "".join(f'    printf("{f} %zu\\n", offsetof(egeria_muon_tensor, {f}));\n' for f, _ in m._fields_) + "    return 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", str(HEADER.parent), str(src), "-o", str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(m)
    for f, _ in m._fields_:
        assert int(got[f]) == getattr(m, f).offset, f


def _matrix(**more):
    t = ops._MuonTensor(param=64, m=64, rows=8, cols=10, param_type=ops.BF16, grad_type=ops.BF16, module=-1, scale=1.0)
    for k, v in more.items():
        setattr(t, k, v)
    return t


def _create(tensors, steps=5, grad=64, workspace=1024, nbytes=1 << 24):
    h = ctypes.c_void_p()
    table = (ops._MuonTensor * max(len(tensors), 1))(*tensors)
    grads = (ctypes.c_void_p * max(len(tensors), 1))(*[grad] * len(tensors))
    return ops.lib().egeria_muon_create(ctypes.byref(h), len(tensors), table, grads, steps, workspace, nbytes)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=-1), dict(param=None), dict(m=None), dict(param_type=3), dict(grad_type=2), dict(module=-2),
                                    dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(scale=float("inf")), dict(param=65), dict(m=66),
                                    dict(master=66)])
def test_refuses_a_bad_matrix(change):
    assert _create([_matrix(**change)]) == eg.ERR_INVALID_ARG


def test_refuses_bad_calls():
    assert _create([]) == eg.ERR_INVALID_ARG
    assert _create([_matrix()], grad=None) == eg.ERR_INVALID_ARG
    assert _create([_matrix()], grad=65) == eg.ERR_INVALID_ARG
    assert _create([_matrix()], steps=0) == eg.ERR_INVALID_ARG
    assert _create([_matrix()], steps=17) == eg.ERR_INVALID_ARG
    assert _create([_matrix()], workspace=None) == eg.ERR_WORKSPACE
    assert _create([_matrix()], workspace=1040) == eg.ERR_WORKSPACE
    assert _create([_matrix()], nbytes=64) == eg.ERR_WORKSPACE
    assert _create([_matrix(rows=2 ** 22 + 1)]) == eg.ERR_UNSUPPORTED_SHAPE
    L, d = ops.lib(), ctypes.c_double
    assert L.egeria_muon_create(None, 1, None, None, 5, None, 0) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_step(None, None, d(1e-3), d(0.9), 1, d(1e-7), None, None) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_set_grads(None, None, None) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_destroy(None) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_device_status(None) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_debug_stall_next(None, 1) == eg.ERR_INVALID_ARG
    assert L.egeria_muon_launch_count(None) == 0


def test_workspace_sizes():
    def size(*shapes, steps=5):
        return ops.lib().egeria_muon_workspace_bytes(len(shapes), (ops._MuonTensor * len(shapes))(*[_matrix(rows=r, cols=c) for r, c in shapes]), steps)

    assert size((8, 8), steps=0) == size((8, 8), steps=17) == size((-1, 8)) == size((2 ** 22 + 1, 8)) == 0
    assert size((0, 8)) > 0
    assert 6 * 1024 * 4096 + 4 * 1024 * 1024 <= size((1024, 4096)) <= 6 * 1024 * 4096 + 4 * 1024 * 1024 + (1 << 18)
    assert size((64, 64)) < size((64, 64), (64, 64)) < size((64, 64), (64, 128))
    assert size((2 ** 63 - 1, 8)) == size((8, 8), (8, 2 ** 63 - 1)) == 0


@pytest.mark.parametrize("second", [dict(param=4096), dict(param=4096 + 158), dict(master=4096), dict(m=8192), dict(m=8192 - 316), dict(m=4096)])
def test_refuses_matrices_that_share_values(second):
    """8 x 10: 160 bytes of weights, 320 of a momentum or a master."""
    first = dict(param=4096, m=8192)
    assert _create([_matrix(**first), _matrix(**{**dict(param=1 << 16, m=1 << 17), **second})]) == eg.ERR_INVALID_ARG


@pytest.mark.parametrize("same", [dict(param=64, m=64), dict(param=64, m=222), dict(param=64, m=1024, master=1024), dict(param=64, m=1024, master=220)])
def test_refuses_a_matrix_that_shares_values_with_itself(same):
    assert _create([_matrix(**{k: v // 4 * 4 for k, v in same.items()})]) == eg.ERR_INVALID_ARG
