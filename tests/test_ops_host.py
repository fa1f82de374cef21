"""CPU-only checks of the training operators' C ABI: exports, header, workspace sizing, refusals."""
import ctypes
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2201_06227_b200 import binding as eg
from paper_2201_06227_b200 import ops

HEADER = Path(__file__).resolve().parent.parent / "include" / "egeria_ops.h"


def test_library_exports_every_declared_operator():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(egeria_[a-z_0-9]+)\s*\(", text)))
    assert sorted(ops.EXPORTS) == names
    for name in names:
        assert hasattr(ops.lib(), name)


def test_struct_has_the_headers_layout(tmp_path):
    """The mirror of egeria_adamw_tensor has the size and the field offsets that a C compiler gives the header's, and the
    header is C99 on its own."""
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    m = ops._AdamTensor
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include "egeria_ops.h"\n#include <stdio.h>\nint main(void) {\n    printf("size %zu\\n", sizeof(egeria_adamw_tensor));\n' +
                   "".join(f'    printf("{f} %zu\\n", offsetof(egeria_adamw_tensor, {f}));\n' for f, _ in m._fields_) + "    return 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", str(HEADER.parent), str(src), "-o", str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got["size"]) == ctypes.sizeof(m)
    for f, _ in m._fields_:
        assert int(got[f]) == getattr(m, f).offset, f


def test_extension_refuses_what_is_no_tensor_or_not_on_the_gpu():
    import torch
    n = ops._native()
    x = torch.zeros(4, 4, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        n.linear_forward(0, 0, 0, 0, x, x, None, 0, None, False)                 # an argument short
    with pytest.raises(ValueError):
        n.linear_forward(0, 0, 0, 0, x, 3, None, 0, None, False, None)
    with pytest.raises(ValueError):
        n.linear_forward(0, 0, 0, 0, x, x, None, 0, None, False, None)           # host memory
    with pytest.raises(ValueError):
        n.linear_backward(0, 0, 0, 0, x, None, None, None, 0, None, 0, True, True, True)
    with pytest.raises(ValueError):
        n.norm_forward(0, 0, 0, 0, x, x, None, None, None, None, None, 0, 0, True, True, 1.0, 1e-5)
    with pytest.raises(ValueError):
        n.norm_backward(0, 0, 0, 0, x, x, x, x, None, None, None, None, None, None, 0, 0, True, True, 1.0, True)
    with pytest.raises(TypeError):
        n.norm_forward(0, 0, 0, 0, x, x, None, None, None, None, None, 0, 0, True, True, "1", 1e-5)
    with pytest.raises(ValueError):
        n.adamw_step(0, 0, 0, 0, 1e-3, 0.9, 0.999, 1e-8, x, None, -1)


def test_workspace_sizes():
    assert ops.egeria_linear_workspace_bytes(0, 64, 64) >= ops.OPS_WORKSPACE_MIN
    assert ops.egeria_linear_workspace_bytes(-1, 64, 64) == 0
    assert ops.egeria_linear_workspace_bytes(1, 0, 64) == 0
    assert ops.egeria_linear_workspace_bytes(1, 64, 2 ** 31) == 0
    # copies of all three operands fit, whatever their alignment
    assert ops.egeria_linear_workspace_bytes(1000, 1001, 999) >= 2 * (1000 * 1008 + 999 * 1008 + 1000 * 1000)
    assert ops.egeria_norm_workspace_bytes(10, 0) == 0
    assert ops.egeria_norm_workspace_bytes(10, ops.NORM_MAX_COLS + 1) == 0
    assert ops.egeria_norm_workspace_bytes(10, ops.NORM_MAX_COLS) > ops.OPS_WORKSPACE_MIN


def _tensor(**more):
    t = ops._AdamTensor(param=64, m=64, v=64, m_scale=64, v_scale=64, n=10, param_type=ops.BF16, grad_type=ops.BF16, module=-1)
    for k, v in more.items():
        setattr(t, k, v)
    return t


def _create(tensors, flags=0, grad=64, steps=64, workspace=1024, nbytes=1 << 20):
    h = ctypes.c_void_p()
    table = (ops._AdamTensor * max(len(tensors), 1))(*tensors)
    grads = (ctypes.c_void_p * max(len(tensors), 1))(*[grad] * len(tensors))
    return ops.lib().egeria_adamw_create(ctypes.byref(h), len(tensors), table, grads, steps, workspace, nbytes, flags)


@pytest.mark.parametrize("change", [dict(n=-1), dict(param=None), dict(m=None), dict(v=None), dict(param_type=3), dict(grad_type=2),
                                    dict(module=-2), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(param=65),
                                    dict(m=66), dict(master=66)])
def test_adamw_refuses_a_bad_tensor(change):
    assert _create([_tensor(**change)]) == eg.ERR_INVALID_ARG


def test_adamw_refuses_bad_calls():
    assert _create([]) == eg.ERR_INVALID_ARG
    assert _create([_tensor()], flags=2) == eg.ERR_INVALID_ARG
    assert _create([_tensor()], grad=None) == eg.ERR_INVALID_ARG
    assert _create([_tensor()], grad=65) == eg.ERR_INVALID_ARG
    assert _create([_tensor()], steps=None) == eg.ERR_INVALID_ARG
    assert _create([_tensor(m_scale=None)], flags=ops.ADAMW_8BIT) == eg.ERR_INVALID_ARG
    assert _create([_tensor()], workspace=None) == eg.ERR_WORKSPACE
    assert _create([_tensor()], workspace=1040) == eg.ERR_WORKSPACE
    assert _create([_tensor()], nbytes=64) == eg.ERR_WORKSPACE
    assert ops.lib().egeria_adamw_workspace_bytes(1, (ops._AdamTensor * 1)(_tensor(n=-1)), 0) == 0
    d = ctypes.c_double
    assert ops.lib().egeria_adamw_step(None, None, d(1e-3), d(0.9), d(0.999), d(1e-8), None, None) == eg.ERR_INVALID_ARG
    assert ops.lib().egeria_adamw_set_grads(None, None, None) == eg.ERR_INVALID_ARG
    assert ops.lib().egeria_adamw_destroy(None) == eg.ERR_INVALID_ARG


def test_null_handles_and_arguments():
    L = ops.lib()
    assert L.egeria_ops_create(None, None, 0) == eg.ERR_INVALID_ARG
    h = ctypes.c_void_p()
    assert L.egeria_ops_create(ctypes.byref(h), None, 1 << 20) == eg.ERR_WORKSPACE
    assert L.egeria_ops_create(ctypes.byref(h), 1024, 100) == eg.ERR_WORKSPACE
    assert L.egeria_ops_create(ctypes.byref(h), 1040, 1 << 20) == eg.ERR_WORKSPACE
    assert L.egeria_ops_destroy(None) == eg.ERR_INVALID_ARG
    assert L.egeria_ops_device_status(None) == eg.ERR_INVALID_ARG
    assert L.egeria_ops_launch_count(None) == 0
    for call in (L.egeria_linear_forward, L.egeria_linear_backward, L.egeria_norm_forward, L.egeria_norm_backward):
        assert call(None, None, bytes(256)) == eg.ERR_INVALID_ARG
        assert call(None, None, None) == eg.ERR_INVALID_ARG
