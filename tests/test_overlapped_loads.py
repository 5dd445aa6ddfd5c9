"""Kernels that may start while the one before them drains (tc::after_previous) read
what that one may still be writing.  Loads of the read-only path are for data that nobody writes
during the kernel, so the sources of these kernels must not ask for them."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_13716_gb300", "csrc")


def code(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


OVERLAPPED = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu"))) if "after_previous()" in code(p)]


def test_there_are_such_kernels():
    assert {os.path.basename(p) for p in OVERLAPPED} >= {"glr.cu", "muon.cu"}


@pytest.mark.parametrize("path", OVERLAPPED, ids=os.path.basename)
def test_no_read_only_loads(path):
    text = code(path)
    assert "__ldg" not in text and "ld.global.nc" not in text and "__restrict__" not in text
