"""Rules of the kernels that no run can show to be kept, read from their sources."""
import os
import re

from paper_2407_00952_b200 import build


def sources():
    for name in sorted(os.listdir(build.CSRC)):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(build.CSRC, name)) as f:
                yield name, re.sub(r"//[^\n]*", "", f.read())


def test_every_bounded_wait_is_looked_at():
    """A wait that ran out returns false: the data is not there, and a kernel that goes on computes with what lay in its place."""
    waits = 0
    for name, text in sources():
        waits += len(re.findall(r"\bmbar_wait(?:_warp)?\(", text))
        ignored = re.findall(r"(?<=[;{})])\s*((?:tc::)?mbar_wait(?:_warp)?\([^;]*;)", text)
        assert not ignored, (name, ignored)
    assert waits > 20
