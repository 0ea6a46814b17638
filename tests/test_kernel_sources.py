"""Rules of the memory model that no run can show to be broken, kept by reading the kernels' sources."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_07306_b200", "csrc")


def sources():
    files = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))
    assert len(files) > 10
    return {os.path.basename(f): open(f).read() for f in files}


def test_arrivals_release_what_was_done_before_them():
    """An arrival that hands a buffer back orders the reads of it before the next writes: a relaxed one orders nothing."""
    for name, text in sources().items():
        assert not re.search(r"mbarrier\.arrive[\w.]*\.relaxed", text), name
