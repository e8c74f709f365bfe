"""Paged calls without a GPU: what the sources promise, and calls of the bookkeeping that change nothing when they fail."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_read_only_loads():
    """The paged kernels begin while the one before may still write tables, lengths and lists, which loads that assume constant
    memory do not allow for."""
    found = glob.glob(os.path.join(ROOT, "paper_2608_14191_gb300", "csrc", "paged*.cu*"))
    assert len(found) >= 4
    for path in found:
        with open(path) as f:
            assert not re.search(r"__ldg\b|ld\.global\.nc|ldu\.global", f.read()), path
