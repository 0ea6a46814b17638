"""C entries that allocate host memory return an error where there is none: kept by reading their source."""
import re

from tests.test_kernel_sources import sources


def test_forward_calls_let_no_exception_through():
    text = sources()["pt_api.cu"]
    for name in ("pt_prefill", "pt_decode_step", "pt_extend", "pt_call_context"):
        body = re.search(r"\npt_status " + name + r"\([^{}]*\) (?:try )?\{.*?\n\}[^\n]*\n", text, re.S).group(0)
        assert ") try {" in body and body.rstrip().endswith("catch (const std::bad_alloc&) {"), name
