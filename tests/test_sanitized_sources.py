"""What the sanitizer builds cover: every source whose host code works out the size of a workspace or the shape of a launch of its own."""
import os
import re

from paper_2010_15884_amd import build


def test_workspaces_are_worked_out_under_the_sanitizers():
    defines = {src for src in build.SOURCES if re.search(r"^size_t \w+_workspace\(", open(os.path.join(build.CSRC, src)).read(), re.M)}
    assert len(defines) >= 4 and defines <= set(build.HOST_LOGIC), defines - set(build.HOST_LOGIC)
