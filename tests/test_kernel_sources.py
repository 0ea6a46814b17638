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


def test_loads_of_tensor_memory_are_waited_for_by_name():
    """To the compiler a tensor-memory load has written its registers where it stands.  The one wait for such loads names them, so
    that no arithmetic on them is moved in front of it; no kernel has a wait of its own, and none discards what it loads."""
    waits = [(name, m.start()) for name, text in sources().items() for m in re.finditer(r"tcgen05\.wait::ld", text)]
    assert [name for name, _ in waits] == ["pt_tmem.cuh"], waits
    text = sources()["pt_tmem.cuh"]
    body = text[waits[0][1]:text.index("}", waits[0][1])]
    assert "tm_pin<N>(v);" in body and '"+f"(v[i])' in text
    for name, text in sources().items():
        loads, named = len(re.findall(r"\bt[mc]_ld(?:16|32)\(", text)), len(re.findall(r"\btm_wait_ld<\d+>\(", text))
        assert (loads > 0) == (named > 0) or name == "pt_tcgen05.cuh", name
