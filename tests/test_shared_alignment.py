"""Dynamic shared memory is read 16 bytes at a time: its declarations say that it is aligned so."""
import glob
import os
import re

import paper_2604_11288_b200 as ta

CSRC = os.path.join(os.path.dirname(ta.__file__), "csrc")


def test_dynamic_shared_memory_is_declared_aligned():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        src = re.sub(r"//[^\n]*", "", open(path).read())
        for align, name in re.findall(r"extern\s+__shared__\s+(?:__align__\((\d+)\)\s+)?[\w ]+?\s*(\w+)\[\]", src):
            found += 1
            rounded_up = re.search(rf"\(uintptr_t\){name} \+ \d+\) & ~", src)
            assert (align and int(align) >= 16) or rounded_up, (os.path.basename(path), name)
    assert found >= 7
