"""What the serving kernels' sources have to keep to, checked on their text: no
run can show it, as a load through the read-only path gives the right value
nearly always."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_07001_gb300", "csrc")


def code_of(path):
    """The file without comments."""
    text = open(path).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def overlapped():
    """The files whose kernels start while their predecessor runs, and the headers they share."""
    files = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))) if "after_previous()" in code_of(p)]
    return files + [os.path.join(CSRC, n) for n in ("paged.cuh", "prompt.cuh", "tc.cuh")]


def test_the_overlapped_kernels_are_found():
    names = {os.path.basename(p) for p in overlapped()}
    assert {"paged.cu", "paged_attention.cu", "prompt.cu", "prompt_f32.cu", "prompt_tc.cu", "serve.cuh"} <= names


@pytest.mark.parametrize("path", overlapped(), ids=os.path.basename)
def test_no_read_only_loads_in_overlapped_kernels(path):
    # A kernel that starts under its predecessor's end, or rotates in place, reads memory that is written
    # during its own life: the read-only path (__ldg, ld.global.nc, const __restrict__ arguments) is not ordered
    # by the wait for the predecessor and need not see those writes.
    code = code_of(path)
    for what in (r"\b__ldg\s*\(", r"ld\.global(\.\w+)*\.nc\b", r"__restrict__"):
        assert not re.search(what, code), f"{os.path.basename(path)}: {what}"
