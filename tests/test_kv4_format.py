"""The 4-bit cache format on the CPU: the oracle's definition against itself, and refusals of the calls (no GPU work)."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv4
from paper_2602_07306_b200 import pt
from tests.test_host_api import lib                           # noqa: F401  (a fixture)

FAKE = C.c_void_p(0x10000)


@pytest.mark.parametrize("dh", [64, 128])
def test_every_place_of_a_block_is_used_once(dh):
    kc, vc, ks, vs, shift = kv4.places(dh)
    nibbles = np.concatenate([(2 * a + (shift > 0)).ravel() for a in (kc, vc)] + [np.stack([2 * a, 2 * a + 1]).ravel() for a in (ks, vs)])
    assert np.array_equal(np.sort(nibbles), np.arange(2 * kv4.block_bytes(dh)))


def test_scales_are_the_upper_half_of_fp16():
    half = (np.arange(256, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
    assert np.array_equal(half[:248], kv4.SCALES) and np.isnan(half[255])


def test_quantised_values():
    x = np.zeros((8, 64))
    x[1, 3] = 6.0                                              # scale 1
    x[2, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]        # ties go to the even code
    x[3, :2] = [6.001, -1]                                     # the next scale, 1.125
    x[4, 0] = 1e30                                             # saturates
    x[5, 40] = np.nan                                          # a group alone is lost
    x[6, 33] = -np.inf
    x[7, :2] = [-0.0, 1e-20]                                   # below the smallest scale
    code, byte = kv4.quantize(x)
    v = kv4.values(code, byte)
    assert byte[0, 0] == 0 and not v[0].any() and byte[1, 0] == 120 and v[1, 3] == 6
    assert v[2, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]
    assert v[3, :2].tolist() == [6.75, -1.125] and v[4, 0] == 6 * 61440
    assert np.isnan(v[5, 32:]).all() and not v[5, :32].any() and byte[6, 1] == 255 and code[6, 33] == 0
    assert byte[7, 0] == 1 and not v[7].any() and code[7, 0] == 8
    rng = np.random.default_rng(0)
    y = rng.standard_normal((100, 128)) * np.exp2(rng.integers(-12, 12, (100, 1)))
    d = np.abs(kv4.values(*kv4.quantize(y)) - y).reshape(100, 4, 32).max(-1)
    assert (d <= np.abs(y).reshape(100, 4, 32).max(-1) * 1.125 / 6 + 2.0 ** -17).all()    # half the largest step of a scale that is 1 + 1/8 too large at most


def test_bytes_hold_the_values():
    rng = np.random.default_rng(1)
    for dh in (64, 128):
        k, v = rng.standard_normal((2, 3, dh)), rng.standard_normal((2, 3, dh))
        pool = np.full((2, 4, 2, 3, 17 * dh), 255, np.uint8)
        for i, (page, slot) in enumerate(((1, 0), (3, 37), (1, 15))):
            kv4.put(pool, page, 1, slot, k[:, i], v[:, i])
        got = kv4.get(pool)
        for i, (page, slot) in enumerate(((1, 0), (3, 37), (1, 15))):
            for w, x in enumerate((k, v)):
                assert np.array_equal(got[:, page, w, 1, slot], kv4.values(*kv4.quantize(x[:, i])))
        assert np.isnan(got[:, 0]).all() and np.isnan(got[:, 1, :, 1, 1:15]).all()


def at(n):
    return C.c_void_p(n)


def test_refusals(lib):
    W = lambda **kw: lib.pt_kernel_kv_write_e2m1(*({"k": FAKE, "v": FAKE, "ts": 8, "rs": 8, "T": 2, "M": 3, "nkv": 2, "dh": 128, "ps": 16, "pages": 4,  # noqa: E731
                                                    "pool": FAKE, "pts": 16, "slots": FAKE, "ko": None, "vo": None, "status": FAKE} | kw).values(), None)
    R = lambda **kw: lib.pt_kernel_kv_read_e2m1(*({"pool": FAKE, "pts": 16, "bt": FAKE, "maxp": 4, "kv": FAKE, "T": 2, "B": 3, "nkv": 2, "dh": 64, "ps": 32, "pages": 4,  # noqa: E731
                                                   "out": FAKE, "ots": 8, "obt": FAKE, "omaxp": 5, "ops": 24, "opages": 7, "status": FAKE} | kw).values(), None)
    n = C.c_size_t()
    assert lib.pt_kernel_attn_e2m1_scratch_bytes(2, 8, 2, 128, C.byref(n)) == 0 and n.value > 0
    A = lambda **kw: lib.pt_kernel_attn_e2m1(*({"q": FAKE, "pool": FAKE, "pts": 16, "bt": FAKE, "maxp": 4, "ql": FAKE, "kv": FAKE, "T": 2, "B": 3, "M": 5, "nq": 8,  # noqa: E731
                                                "nkv": 2, "dh": 128, "ps": 16, "pages": 4, "out": out, "scratch": FAKE, "bytes": n.value, "status": FAKE} | kw).values(), None)
    odd = at(0x10004)
    out = at(0x20000)
    for call, refused in (
            (W, [(1, dict(k=None)), (1, dict(slots=None)), (1, dict(status=None)), (1, dict(ko=FAKE)), (1, dict(M=0)), (1, dict(T=0)), (1, dict(ts=-8)), (1, dict(rs=-8)),
                 (1, dict(pages=0)), (1, dict(nkv=0)), (3, dict(dh=32)), (3, dict(dh=96)), (3, dict(ps=8)), (3, dict(ps=24)), (3, dict(ps=80)), (3, dict(T=70000)),
                 (6, dict(pool=odd)), (6, dict(pts=8)), (6, dict(k=odd)), (6, dict(v=odd)), (6, dict(ko=odd, vo=FAKE)), (6, dict(ts=4)), (6, dict(rs=12)),
                 (6, dict(slots=odd)), (6, dict(status=at(0x10002)))]),
            (R, [(1, dict(out=None)), (1, dict(obt=None)), (1, dict(kv=None)), (1, dict(B=0)), (1, dict(maxp=0)), (1, dict(omaxp=0)), (1, dict(opages=0)), (1, dict(ots=-8)),
                 (1, dict(ops=12)), (1, dict(ops=72)), (1, dict(pts=-16)), (3, dict(dh=32)), (3, dict(ps=40)), (3, dict(maxp=1 << 27)), (3, dict(omaxp=1 << 28)), (3, dict(B=1 << 20, maxp=1 << 20)),
                 (6, dict(out=odd)), (6, dict(ots=4)), (6, dict(pool=odd)), (6, dict(bt=at(0x10002))), (6, dict(kv=at(0x10002)))]),
            (A, [(1, dict(q=None)), (1, dict(out=FAKE)), (3, dict(T=65536)), (3, dict(T=60000, nkv=500, nq=500)), (1, dict(kv=None)), (1, dict(scratch=None)), (1, dict(B=0)), (1, dict(M=0)), (1, dict(M=(1 << 26) + 1)), (1, dict(nq=7)), (1, dict(nq=0)),
                 (1, dict(ql=None)), (1, dict(maxp=0)), (3, dict(nq=18)), (3, dict(dh=32)), (3, dict(ps=8)), (3, dict(maxp=1 << 27)), (4, dict(bytes=n.value - 1)),
                 (3, dict(B=1 << 20, M=1 << 20, maxp=1 << 20)), (6, dict(q=odd)), (6, dict(out=odd)), (6, dict(scratch=at(0x10080))), (6, dict(pool=odd)), (6, dict(pts=24)), (6, dict(ql=at(0x10002)))])):
        for code, kw in refused:
            assert call(**kw) == code, (call, kw, lib.pt_last_error())
    assert lib.pt_kernel_attn_e2m1_scratch_bytes(2, 8, 2, 96, C.byref(n)) == 1


class Cuda:
    """A tensor of the CPU that says it is a CUDA device's."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, t, index=0):
        self.t, self.index = t, index

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, i):
        return Cuda(self.t[i], self.index)


def test_the_binding_checks_shapes_types_and_devices(monkeypatch):
    import torch
    launched = []
    monkeypatch.setattr(pt, "_call", lambda index, fn, *args: launched.append(args))
    bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    z = lambda *s, dtype=bf: Cuda(torch.zeros(s, dtype=dtype))                       # noqa: E731
    shape = dict(nkv=2, dh=64, ps=32)
    pool, status = z(2, 3, 2, 2, 17 * 64, dtype=u8), z(16, dtype=i32)
    n = C.c_size_t()
    assert pt.lib().pt_kernel_attn_e2m1_scratch_bytes(2, 4, 2, 64, C.byref(n)) == 0
    write = dict(k=z(2, 5, 128), v=z(2, 5, 128), pool_l=pool, slots=z(5, dtype=torch.int64), k_out=None, v_out=None, status=status)
    read = dict(pool_l=pool, block_table=z(4, 2, dtype=i32), kv_len=z(4, dtype=i32), out=z(2, 6, 2, 2, 8, 64), out_table=z(4, 9, dtype=i32), status=status)
    attn = dict(q=z(2, 5, 256), pool_l=pool, block_table=z(4, 2, dtype=i32), kv_len=z(4, dtype=i32), q_len=z(4, dtype=i32), nq=4, out=z(2, 5, 256),
                scratch=z(n.value, dtype=u8), status=status)
    other = lambda t: Cuda(t.t, 1)                                                   # noqa: E731
    for fn, good, bad in (
            (pt.kernel_kv_write_e2m1, write, [dict(k=z(2, 5, 128, dtype=torch.float32)), dict(v=z(2, 5, 64)), dict(k=z(2, 5, 130)[:, :, :128]), dict(slots=z(5, dtype=i32)),
                                              dict(slots=z(4, dtype=torch.int64)), dict(k_out=z(2, 5, 128)), dict(pool_l=z(2, 3, 2, 2, 1000, dtype=u8)), dict(pool_l=z(1, 3, 2, 2, 17 * 64, dtype=u8)),
                                              dict(pool_l=other(pool)), dict(v=other(z(2, 5, 128))), dict(slots=Cuda(torch.zeros(10, dtype=torch.int64)[::2])),
                                              dict(k_out=z(2, 5, 128), v_out=z(5, 2, 128)), dict(status=z(8, dtype=i32)), dict(pool_l=Cuda(pool.t.transpose(1, 2)))]),
            (pt.kernel_kv_read_e2m1, read, [dict(out=z(2, 6, 2, 1, 8, 64)), dict(out=z(2, 6, 2, 2, 8, 128)), dict(out=z(2, 6, 2, 2, 8, 64, dtype=torch.float16)), dict(kv_len=z(3, dtype=i32)),
                                            dict(out_table=z(3, 9, dtype=i32)), dict(block_table=z(4, 2, dtype=torch.int64)), dict(out=other(read["out"])), dict(kv_len=other(read["kv_len"])),
                                            dict(out=Cuda(read["out"].t.transpose(1, 2).contiguous().transpose(1, 2)))]),
            (pt.kernel_attn_e2m1, attn, [dict(q=z(2, 5, 128)), dict(q=z(2, 5, 256, dtype=torch.float16)), dict(q_len=z(3, dtype=i32)), dict(block_table=z(3, 2, dtype=i32)),
                                         dict(out=z(2, 4, 256)), dict(scratch=other(attn["scratch"])), dict(status=other(status)), dict(pool_l=z(3, 3, 2, 2, 17 * 64, dtype=u8)),
                                         dict(q=Cuda(torch.zeros((2, 10, 256), dtype=bf)[:, ::2])), dict(kv_len=Cuda(torch.zeros(8, dtype=i32)[::2]))])):
        before = len(launched)
        fn(**good, **shape)
        assert len(launched) == before + 1
        for kw in bad:
            with pytest.raises((ValueError, RuntimeError)):
                fn(**(good | kw), **shape)
        assert len(launched) == before + 1


def test_cache_layout_and_offsets(lib):
    cfg = pt.pt_config(2, 2, 4, 512, 4, 2, 352, 10000.0, 1e-6, pt.PT_BF16, 0, 900, 0, 0, 0)
    h, c = C.c_void_p(), C.c_void_p()
    assert lib.pt_model_create(C.byref(cfg), C.byref(h)) == 0
    n, m = C.c_size_t(), C.c_size_t()
    pages, ps, dh = 7, 32, 128
    assert lib.pt_kv_cache_bytes_ex(h, pages, ps, pt.PT_KV_E2M1, C.byref(n)) == 0
    assert n.value == 2 * 4 * pages * 2 * (ps // 16) * kv4.block_bytes(dh)
    assert lib.pt_kv_cache_bytes_ex(h, pages, 24, pt.PT_KV_E2M1, C.byref(m)) == 3
    assert lib.pt_kv_cache_bytes_ex(h, pages, ps, 3, C.byref(m)) == 1
    assert lib.pt_kv_cache_alloc_ex(h, pages, ps, pt.PT_KV_E2M1, FAKE, n.value - 1, C.byref(c)) == 4
    assert lib.pt_kv_cache_alloc_ex(h, pages, ps, pt.PT_KV_E2M1, FAKE, n.value, C.byref(c)) == 0
    assert lib.pt_kv_seq_reserve(c, 5, 100) == 0
    off, sc = C.c_int64(), C.c_int64()
    blk = kv4.block_bytes(dh)
    for track, layer, pos, kv, head in ((0, 0, 0, 0, 0), (1, 3, 99, 1, 1), (0, 2, 47, 0, 1), (1, 0, 16, 1, 0)):
        assert lib.pt_kv_slot(c, track, layer, 5, pos, kv, head, C.byref(off)) == 0
        assert lib.pt_kv_scale_slot(c, track, layer, 5, pos, kv, head, C.byref(sc)) == 0
        want = ((((track * 4 + layer) * pages + pos // ps) * 2 + head) * 2 + pos % ps // 16) * blk + kv * blk // 2
        assert off.value == want and sc.value == want + 8 * dh
    # workspace: one for this format serves the others
    sizes = []
    for d in (pt.PT_KV_MODEL, pt.PT_KV_E4M3, pt.PT_KV_E2M1):
        assert lib.pt_workspace_bytes_ex(h, 64, 2, 16, d, 500, C.byref(m)) == 0
        e = C.c_size_t()
        assert lib.pt_extend_workspace_bytes(h, 64, 2, 16, d, 500, C.byref(e)) == 0
        sizes.append((m.value, e.value))
    assert sizes[0] < sizes[1] < sizes[2] and sizes[0][1] < sizes[1][1] < sizes[2][1]
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)
    for bad in (dict(dtype=pt.PT_F32), dict(flags=1), dict(heads=16, kv=8)):      # fp32, the plain kernels, head_dim 32
        cfg = pt.pt_config(2, 2, 4, 512, bad.get("heads", 4), bad.get("kv", 2), 352, 10000.0, 1e-6, bad.get("dtype", pt.PT_BF16), 0, 900, bad.get("flags", 0), 0, 0)
        assert lib.pt_model_create(C.byref(cfg), C.byref(h)) == 0
        assert lib.pt_kv_cache_bytes_ex(h, pages, ps, pt.PT_KV_E2M1, C.byref(n)) == 3
        lib.pt_model_destroy(h)
