"""What the compiler cannot check in the kernels' sources: rules that a mistake
would break without failing a run here."""
import glob
import os
import re
import struct

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


def test_shared_counts_change_behind_a_barrier():
    """All waves branch on the counts of a row's workgroup, so between one reading and the next
    store there is a barrier, in the function that stores."""
    sample = text(os.path.join(CSRC, "sample.hip"))
    stores = list(re.finditer(r"sh\.(count|groups)\s*=(?!=)", sample))
    assert len(stores) >= 4
    for m in stores:
        before = sample[sample.rfind("__device__", 0, m.start()):m.start()]
        assert "__syncthreads()" in before, sample[m.start() - 200:m.end() + 20]
        assert f"sh.{m[1]}" not in before[before.rfind("__syncthreads()"):], before[-200:]


def test_sampling_chunk_without_logits():
    """The N of a chunk with nothing to take lies between the x of what is never taken, whose
    exponent is held from below only before it becomes an integer, and that of every logit."""
    sample = text(os.path.join(CSRC, "sample.hip"))
    absent = struct.unpack("<d", struct.pack("<Q", (int(re.search(r"kFar = (0x[0-9a-f]+)", sample)[1], 16) | 1 << 31) << 32))[0]
    none = re.search(r"largest == 0 \? (\S+) :", sample)[1]
    none = re.search(rf"\b{none} = (\S+);", sample)[1] if none.startswith("k") else none
    least = -3.4028235e38 * 1.4426950408889634 / 2.0 ** -149
    assert absent < float(none) - 1e6 < least - 1e6, (absent, none, least)
