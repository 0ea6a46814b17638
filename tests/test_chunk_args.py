"""Refusals of chunk attention beyond its plain ranges (no GPU work)."""
import ctypes as C

import pytest

from paper_2602_07306_b200 import pt
from tests.test_host_api import lib                           # noqa: F401  (a fixture)

FAKE = C.c_void_p(0x10000)


def test_tables_of_more_keys_than_32_bits_count_in_tiles(lib):
    """Key numbers are rounded up to tiles of 128 in 32 bits."""
    n = C.c_size_t()
    assert lib.pt_kernel_chunk_attn_scratch_bytes(2, 3, 8, 128, C.byref(n)) == 0
    for impl, maxp, ps in ((0, (1 << 27), 16), (1, (1 << 27), 16), (0, (1 << 31) // 64, 64), (1, (1 << 31) // 40, 40), (1, 0x7fffffff, 64)):
        rc = lib.pt_kernel_chunk_attn(FAKE, FAKE, 1 << 20, FAKE, maxp, FAKE, FAKE, 2, 3, 5, 8, 2, 128, ps, 9, FAKE, impl, FAKE, n.value, FAKE, None)
        assert rc == 3 and b"keys" in lib.pt_last_error(), (impl, maxp, ps, rc)
