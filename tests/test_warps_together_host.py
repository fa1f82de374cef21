"""CPU-only: every instruction that PTX calls `.aligned`, which a warp has to reach with its lanes together, stands behind a
`__syncwarp()` of its own.  What the compiler happens to bring together is no ground to stand on, and a warp that arrives in
parts is undefined."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2201_06227_b200" / "csrc"
SOURCES = sorted([*CSRC.rglob("*.cuh"), *CSRC.rglob("*.cu")])
# (bar.sync and bar.red are barrier.sync.aligned and barrier.red.aligned)
ALIGNED = re.compile(r'"[^"\n]*(?:\.aligned\b|\bbar\.(?:sync|red)\b)')


def lonely(text):
    """Lines whose aligned instruction has no __syncwarp() between the `{` of its function (or lambda) and itself."""
    bad = []
    for m in ALIGNED.finditer(text):
        depth, i = 0, text.rfind("asm", 0, m.start())
        begin = i
        while begin > 0:
            begin -= 1
            if text[begin] == "}":
                depth += 1
            elif text[begin] == "{":
                line = text[text.rfind("\n", 0, begin) + 1:begin]
                if depth == 0 and (line.rstrip().endswith("]") or not line[:1].isspace()):
                    break
                depth = max(0, depth - 1)
        if "__syncwarp();" not in text[begin:i]:
            bad.append(text.count("\n", 0, m.start()) + 1)
    return bad


@pytest.mark.parametrize("path", SOURCES, ids=lambda p: p.name)
def test_aligned_instructions_meet_first(path):
    assert lonely(path.read_text()) == []


def test_the_scan_sees_what_it_looks_for():
    assert sum(len(ALIGNED.findall(p.read_text())) for p in SOURCES) >= 12
    assert lonely('void f() {\n    if (x) y();\n    asm volatile("tcgen05.wait::ld.sync.aligned;");\n}\n') == [3]
    assert lonely('void f() {\n    __syncwarp();\n    asm volatile("bar.sync 1, 32;");\n}\n') == []
