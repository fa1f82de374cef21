"""The first call for a gated block of a process may be a captured one."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = """
import torch
from paper_2201_06227_b200 import ops
rows, back = {rows}, {back}
g = torch.Generator(device="cuda")
g.manual_seed(1)
t = lambda *s: (torch.randn(*s, generator=g, device="cuda") / 8).bfloat16()
x, w = t(rows, 64), dict(w_gate=t(96, 64), w_up=t(96, 64), w_down=t(64, 96))
pg, pu = t(rows, 96), t(rows, 96)
o = ops.Ops(ops.egeria_gated_workspace_bytes(rows, 64, 96, 64))
before = o.egeria_linear_forward(x, w["w_gate"])
call = (lambda: o.egeria_gated_backward(x, x, **w, g=pg, u=pu)["dx"]) if back else (lambda: o.egeria_gated_forward(x, **w))
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = call()
graph.replay()
torch.cuda.synchronize()
first = y.clone()
assert torch.isfinite(first).all() and first.any()
assert torch.equal(first, call())
o.check_device_status()
print("same")
"""


@pytest.mark.parametrize("rows,back", [(3, False), (70, False), (70, True)])
def test_the_first_call_may_be_captured(rows, back):
    r = subprocess.run([sys.executable, "-c", SCRIPT.format(rows=rows, back=back)], capture_output=True, text=True,
                       cwd=str(Path(__file__).resolve().parent.parent))
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stdout + r.stderr[-2000:]
