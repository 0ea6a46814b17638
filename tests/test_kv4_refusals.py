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


def at(n):
    return C.c_void_p(n)


def test_memory_that_is_written_twice_or_read_as_it_is_written(lib):
    n, A0, B0 = C.c_size_t(), 1 << 20, 1 << 24
    assert lib.pt_kernel_attn_e2m1_scratch_bytes(2, 8, 2, 128, C.byref(n)) == 0

    def attn(q, out):                                          # 2 tracks x 5 rows x 8 heads of 128: 20480 bytes
        return lib.pt_kernel_attn_e2m1(at(q), at(B0), 1 << 20, at(B0), 4, at(B0), at(B0), 2, 3, 5, 8, 2, 128, 16, 4, at(out), at(B0), n.value, at(B0), None)
    for d in (16, 20464, -16, -20464):
        assert attn(A0, A0 + d) == 1 and b"overlap" in lib.pt_last_error()

    def write(k, v, ko, vo, ts=4 * 256, rs=256, pts=1 << 20):  # 2 tracks x 4 rows x 2 heads of 128: 4096 bytes
        return lib.pt_kernel_kv_write_e2m1(at(k), at(v), ts, rs, 2, 4, 2, 128, 16, 4, at(B0), pts, at(B0), at(ko), at(vo), at(B0), None)
    far, out = A0 + (1 << 18), A0 + 8192
    for a in ((A0, far, A0 + 16, far + 16), (A0, far, A0 + 4080, out), (A0, far, out, far - 4080), (A0, far, out, out), (A0, far, out, out + 4080)):
        assert write(*a) == 1, a
    assert write(A0, far, A0, far, rs=264) == 1 and write(A0, far, A0, far, ts=0) == 1
    assert write(A0, far, out, far + 8192, pts=4 * 2 * 17 * 128 - 16) == 1 and b"tracks overlap" in lib.pt_last_error()

    def read(ots):
        return lib.pt_kernel_kv_read_e2m1(at(B0), 0, at(B0), 4, at(B0), 2, 3, 2, 64, 32, 4, at(A0), ots, at(B0), 5, 24, 7, at(B0), None)
    assert read(7 * 2 * 2 * 24 * 64 - 8) == 1 and read(0) == 1
