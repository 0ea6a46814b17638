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


class Cuda:
    """A tensor of the CPU that says it is device 0's."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, i):
        return Cuda(self.t[i])


def test_scratch_and_status_are_whole_blocks_of_memory(monkeypatch):
    """A view with gaps has fewer bytes of its own than the kernel writes behind its first."""
    import torch
    launched = []
    monkeypatch.setattr(pt, "_call", lambda index, fn, *args: launched.append(args))
    i32 = dict(dtype=torch.int32)
    q, pool = torch.zeros((1, 2, 128), dtype=torch.bfloat16), torch.zeros((1, 3, 2, 1, 16, 128), dtype=torch.bfloat16)
    args = [Cuda(t) for t in (q, pool, torch.zeros((1, 2), **i32), torch.zeros(1, **i32), torch.zeros(1, **i32))]
    n = C.c_size_t()
    assert pt.lib().pt_kernel_chunk_attn_scratch_bytes(1, 1, 1, 128, C.byref(n)) == 0

    def go(scratch=torch.zeros(n.value, dtype=torch.uint8), status=torch.zeros(16, **i32)):
        pt.kernel_chunk_attn(*args, nq=1, nkv=1, dh=128, ps=16, out=Cuda(torch.zeros_like(q)), scratch=Cuda(scratch), status=Cuda(status))
    go()
    assert len(launched) == 1
    with pytest.raises(AssertionError):
        go(scratch=torch.zeros(2 * n.value, dtype=torch.uint8)[::2])
    with pytest.raises(AssertionError):
        go(status=torch.zeros(32, **i32)[::2])
    assert len(launched) == 1
