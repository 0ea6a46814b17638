"""Calls of the 4-bit cache's operators at the edge of what they take (no GPU work)."""
import ctypes as C

import torch

from paper_2602_07306_b200 import pt
from tests.test_host_api import lib                           # noqa: F401  (a fixture)
from tests.test_kv4_format import Cuda


def z(*s, dtype=torch.bfloat16):
    return Cuda(torch.zeros(s, dtype=dtype))


def test_calls_of_nothing_launch_nothing(monkeypatch):
    """No rows to write, no sequences to read, no rows to attend: all three return, none calls the library."""
    launched = []
    monkeypatch.setattr(pt, "_call", lambda index, fn, *args: launched.append(args))
    i32, shape = torch.int32, dict(nkv=2, dh=64, ps=32)
    pool, status, none = z(2, 3, 2, 2, 17 * 64, dtype=torch.uint8), z(16, dtype=i32), z(0, dtype=i32)
    pt.kernel_kv_write_e2m1(z(2, 0, 128), z(2, 0, 128), pool, z(0, dtype=torch.int64), status=status, **shape)
    out = z(2, 6, 2, 2, 8, 64)
    assert pt.kernel_kv_read_e2m1(pool, z(0, 2, dtype=i32), none, out, z(0, 9, dtype=i32), status=status, **shape) == (out, status)
    empty = z(2, 0, 256)
    assert pt.kernel_attn_e2m1(empty, pool, z(0, 2, dtype=i32), none, none, nq=4, out=empty, scratch=z(1 << 20, dtype=torch.uint8), status=status, **shape) == (empty, status)
    assert not launched
