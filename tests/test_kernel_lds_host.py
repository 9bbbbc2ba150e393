"""Lanes of a wave that exchange values through LDS say so to the compiler, which may otherwise move a lane's read past another's write."""
import os
import re

from paper_1606_05688_amd import build


def test_a_wave_meets_between_its_writes_and_its_reads():
    """Where a product ends, a wave's rows go through its own part of LDS, 32 at a time: written, read by other lanes, written again."""
    text = open(os.path.join(build.CSRC, "linear.hip")).read()
    start = text.index("float4* const mine")
    end = text[start:text.index("\n}\n", start)]
    steps = re.findall(r"(mine\[[^;]*?\]\s*=[^=])|(=\s*mine\[)|(wave_meets\(\);)", end)
    assert ["write" if w else "read" if r else "meet" for w, r, _ in steps] == ["write", "meet", "read", "meet"]
    # both inside the loop over the rows
    body = end[end.index("for (int j = 0; j < MB; ++j)"):]
    assert body.count("wave_meets();") == 2
