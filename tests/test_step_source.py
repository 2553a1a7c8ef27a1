"""What the compiler cannot check in the kernels' sources: rules that a mistake
would break without failing a run here."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_00916_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.hpp")))


def text(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_dynamic_lds_is_aligned_for_vectors(path):
    """An LDS array of a size given at the launch begins wherever the static ones end, at the
    alignment it is declared with; all of them are read by 16 bytes."""
    for decl in re.findall(r"extern\s+__shared__[^;]*;", text(path)):
        assert "aligned(16)" in decl or "alignas(16)" in decl, decl
