"""Cluster barriers in their .aligned form want the whole warp at the instruction, and
nothing else brings the lanes together after a branch that one of them took: each is
preceded by __syncwarp() in the function that holds it."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2608_01784_gb300" / "csrc"


@pytest.mark.parametrize("path", sorted(CSRC.glob("*.cu*")), ids=lambda p: p.name)
def test_warps_meet_before_aligned_barriers(path):
    text = re.sub(r"//[^\n]*", "", path.read_text())
    for m in re.finditer(r"barrier\.cluster\.arrive[.\w]*\.aligned", text):
        asm = text.rindex("asm", 0, m.start())
        before = text[:asm].rstrip()
        assert before.endswith("__syncwarp();"), text[max(0, asm - 200):m.end()]
