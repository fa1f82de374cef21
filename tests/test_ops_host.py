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


def test_structs_have_the_headers_layout(tmp_path):
    """Every mirror of a struct has the size and the field offsets that a C compiler gives the header's."""
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    def mirror(fields):
        return type("Mirror", (ctypes.Structure,), {"_fields_": fields})

    mirrors = {"egeria_linear_forward_args": mirror(ops._LINEAR_FORWARD), "egeria_linear_backward_args": mirror(ops._LINEAR_BACKWARD),
               "egeria_norm_forward_args": mirror(ops._NORM_FORWARD), "egeria_norm_backward_args": mirror(ops._NORM_BACKWARD),
               "egeria_adamw_tensor": ops._AdamTensor}
    lines = ['#include "egeria_ops.h"', "#include <stdio.h>", "int main(void) {"]
    for name, m in mirrors.items():
        lines.append(f'    printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'    printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in m._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["    return 0;", "}", ""]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", str(HEADER.parent), str(src), "-o", str(exe)], check=True)
    got = dict(line.rsplit(" ", 1) for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, m in mirrors.items():
        assert int(got[name]) == ctypes.sizeof(m)
        for f, _ in m._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(m, f).offset, (name, f)
    # and the packed forms put the values there
    for pack, name in ((ops._pack_linear_forward, "egeria_linear_forward_args"), (ops._pack_linear_backward, "egeria_linear_backward_args"),
                       (ops._pack_norm_forward, "egeria_norm_forward_args"), (ops._pack_norm_backward, "egeria_norm_backward_args")):
        m = mirrors[name]
        values = list(range(1, len(m._fields_) + 1))
        read = m.from_buffer_copy(pack(*values).ljust(ctypes.sizeof(m), b"\0"))
        assert [getattr(read, f) for f, _ in m._fields_] == values


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
    assert ops.lib().egeria_adamw_step(None, None, 1e-3, 0.9, 0.999, 1e-8, None, None) == eg.ERR_INVALID_ARG
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
