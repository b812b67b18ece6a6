"""Rules that the CUDA sources keep, read from the sources: no device is needed."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1901_08924_b200", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))


def _code(path):
    text = open(path).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_what_an_earlier_kernel_writes_is_read_behind_the_wait(path):
    # Kernels start while the one before them in the stream still runs, and wait for it before they touch its data.  A load that claims that nobody writes its
    # data while the kernel lives, or one in assembly that is not volatile, may move in front of that wait.
    code = _code(path)
    assert "__ldg" not in code and "ldg_nc" not in code
    assert not re.search(r"\bld\.global[\w.:]*\.nc\b", code)
    for volatile, text in re.findall(r"\basm\s*(volatile)?\s*\(\s*((?:\"[^\"]*\"\s*)+)", code):
        assert volatile or not re.search(r"\b(ld|st|cp|atom|red)\.", text), text
