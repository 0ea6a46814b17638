"""Host-side logic of the serving entry points (no GPU work): sharing of cache pages between sequences against a brute-force
count of owners, and the refusals of sampling, page copies, chunk attention and ragged calls."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07306_b200 import pt
from tests.test_host_api import _cache, lib, make            # noqa: F401  (lib is a fixture)

FAKE = C.c_void_p(0x10000)


def i32(a):
    return (C.c_int32 * len(a))(*a)


def pages_of(lib, c, seq):
    n = C.c_int32()
    assert lib.pt_kv_block_table(c, seq, None, 0, C.byref(n)) == 0
    buf = (C.c_int32 * max(1, n.value))()
    lib.pt_kv_block_table(c, seq, buf, n.value, C.byref(n))
    return list(buf[:n.value])


def free_pages(lib, c):
    n = C.c_int32()
    assert lib.pt_kv_free_pages(c, C.byref(n)) == 0
    return n.value


def refs(lib, c, page):
    n = C.c_int32()
    assert lib.pt_kv_page_refs(c, page, C.byref(n)) == 0
    return n.value


def test_fork_shares_pages_and_release_frees_the_last_owner(lib):
    rc, h = make(lib)
    pages, ps = 40, 8
    c, _ = _cache(lib, h, pages, ps)
    rng = np.random.default_rng(0)
    alive = {}
    nxt = 0
    for step in range(300):
        op = rng.integers(0, 4)
        if op == 0 or not alive:
            want = int(rng.integers(0, 5 * ps))
            rc = lib.pt_kv_seq_reserve(c, nxt, want)
            if rc == 0:
                alive[nxt] = pages_of(lib, c, nxt)
                assert len(alive[nxt]) == -(-want // ps)
            else:
                assert rc == 5 and -(-want // ps) > free_pages(lib, c)
            nxt += 1
        elif op == 1:
            src = int(rng.choice(list(alive)))
            # nothing was forwarded: every sequence's length is 0, so a fork of length 0 owns no page
            assert lib.pt_kv_seq_fork(c, src, nxt, 0) == 0 and pages_of(lib, c, nxt) == []
            assert lib.pt_kv_seq_fork(c, src, nxt, 0) == 10 and lib.pt_kv_seq_fork(c, src, src, 0) == 10
            assert lib.pt_kv_seq_fork(c, src, nxt + 1, 1) == 1
            alive[nxt] = []
            nxt += 1
        else:
            s = int(rng.choice(list(alive)))
            assert lib.pt_kv_seq_release(c, s) == 0
            del alive[s]
        owners = np.bincount(sum(alive.values(), []), minlength=pages)
        assert [refs(lib, c, p) for p in range(pages)] == owners.tolist()
        assert free_pages(lib, c) == int((owners == 0).sum())
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)


def test_cache_refusals(lib):
    rc, h = make(lib)
    c, nbytes = _cache(lib, h, 6, 8)
    n = C.c_int32()
    assert lib.pt_kv_seq_fork(None, 0, 1, 0) == 1 and lib.pt_kv_seq_fork(c, 0, 1, 0) == 10
    assert lib.pt_kv_seq_reserve(c, 0, 20) == 0
    assert lib.pt_kv_seq_fork(c, 0, -1, 0) == 1 and lib.pt_kv_seq_fork(c, 0, 1, -1) == 1 and lib.pt_kv_seq_fork(c, 0, 1, 1) == 1
    assert lib.pt_kv_page_refs(c, 6, C.byref(n)) == 1 and lib.pt_kv_page_refs(c, -1, C.byref(n)) == 1 and lib.pt_kv_free_pages(c, None) == 1
    # already packed at the front: nothing to copy, the free list becomes ascending
    moved = C.c_int32(-1)
    assert lib.pt_kv_compact(c, C.byref(moved), None) == 0 and moved.value == 0 and pages_of(lib, c, 0) == [0, 1, 2]
    need = C.c_size_t()
    assert lib.pt_kv_cache_bytes(h, 3, 8, C.byref(need)) == 0
    far = C.c_void_p(0x10000 + ((nbytes + 255) // 256 + 1) * 256)
    assert lib.pt_kv_move_pool(c, 3, far, need.value - 1, None) == 4
    assert lib.pt_kv_move_pool(c, 3, C.c_void_p(far.value + 16), need.value, None) == 6
    assert lib.pt_kv_move_pool(c, 3, C.c_void_p(0x10100), need.value, None) == 1 and b"overlap" in lib.pt_last_error()
    assert lib.pt_kv_move_pool(c, 0, far, need.value, None) == 1
    assert lib.pt_kv_cache_bytes(h, 2, 8, C.byref(need)) == 0
    assert lib.pt_kv_move_pool(c, 2, far, need.value, None) == 5
    assert pages_of(lib, c, 0) == [0, 1, 2] and free_pages(lib, c) == 3
    assert lib.pt_kv_seq_release(c, 0) == 0
    assert lib.pt_kv_move_pool(c, 2, far, need.value, None) == 0 and free_pages(lib, c) == 2        # nothing in use: no copy
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)


def test_page_copy_refusals(lib):
    def go(src, dst, sp=4, dp=4, slabs=2, pb=512, a=0x10000, b=0x10000, n=None):
        return lib.pt_kernel_kv_copy_pages(C.c_void_p(a), sp, C.c_void_p(b), dp, slabs, pb, C.cast(i32(src), C.c_void_p), C.cast(i32(dst), C.c_void_p),
                                           len(src) if n is None else n, None)
    assert go([0], [4]) == 1 and go([4], [0]) == 1 and go([-1], [0]) == 1 and go([0], [-1]) == 1
    assert go([0, 1], [2, 2]) == 1 and b"written twice" in lib.pt_last_error()
    assert go([0, 2], [2, 3]) == 1 and b"read and written" in lib.pt_last_error()
    assert go([1], [1]) == 1
    assert go([0], [1], pb=8) == 1 and go([0], [1], pb=520) == 1 and go([0], [1], slabs=0) == 1 and go([0], [1], n=-1) == 1
    assert go([0], [1], a=0x10008, b=0x10008) == 6
    assert go([0], [1], dp=5) == 1                                                                 # one pool, two page counts
    assert go([0], [1], b=0x10000 + 2 * 4 * 512 - 16) == 1 and b"overlap" in lib.pt_last_error()
    assert go([], []) == 0
    assert lib.pt_kernel_kv_copy_pages(None, 4, FAKE, 4, 2, 512, None, None, 0, None) == 1


def test_sizes_that_overflow_and_pointers_off_their_type_are_refused(lib):
    ids = [C.cast(i32([i]), C.c_void_p) for i in (0, 1)]
    for slabs, pages, pb in ((1 << 62, 4, 512), (1 << 40, 1 << 30, 1 << 29), ((1 << 63) - 1, 2, 16)):
        assert lib.pt_kernel_kv_copy_pages(FAKE, pages, FAKE, pages, slabs, pb, ids[0], ids[1], 1, None) == 1 and b"2^62" in lib.pt_last_error()
    odd = C.c_void_p(0x10002)
    for i in range(5, 12):                                        # u, temperature, top_k, top_p, min_p, token, prob
        args = [FAKE, 0, 10, 3, 10, FAKE, None, None, None, None, FAKE, None, None]
        args[i] = odd
        assert lib.pt_sample(*args) == 6, i
    n = C.c_size_t()
    assert lib.pt_kernel_chunk_attn_scratch_bytes(2, 3, 8, 128, C.byref(n)) == 0
    for i in (3, 5, 6, 19):                                       # block_table, q_len, kv_len, status
        args = [FAKE, FAKE, 1 << 20, FAKE, 4, FAKE, FAKE, 2, 3, 5, 8, 2, 128, 16, 9, FAKE, 0, FAKE, n.value, FAKE, None]
        args[i] = odd
        assert lib.pt_kernel_chunk_attn(*args) == 6, i
    rc, h = make(lib, dtype=pt.PT_BF16)
    c, _ = _cache(lib, h, 6, 16, esz=2)
    for f in ("u", "temperature", "top_k", "top_p", "min_p", "prob"):
        sp = pt.pt_sampling(u=FAKE.value)
        setattr(sp, f, odd.value)
        assert lib.pt_generate_sample(h, c, FAKE, 1, 4, 2, i32([0]), C.byref(sp), FAKE, None, FAKE, 1 << 30, None) == 6, f
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)


def test_python_page_numbers_are_not_cut():
    assert pt._page_ids([]).dtype == np.int32 and pt._page_ids(range(3)).tolist() == [0, 1, 2]
    assert pt._page_ids(np.array([5.0, 7.0])).tolist() == [5, 7]
    for bad in (np.array([2 ** 32 + 1]), np.array([0.5]), [1.25, 2]):
        with pytest.raises(ValueError):
            pt._page_ids(bad)


def test_sample_refusals(lib):
    def go(logits=FAKE, dtype=0, stride=10, n=3, vocab=10, u=FAKE, token=FAKE):
        return lib.pt_sample(logits, dtype, stride, n, vocab, u, None, None, None, None, token, None, None)
    assert go(logits=None) == 1 and go(u=None) == 1 and go(token=None) == 1
    assert go(dtype=2) == 1 and go(n=0) == 1 and go(n=(1 << 24) + 1) == 1 and go(vocab=0) == 1 and go(stride=9) == 1
    assert go(vocab=393217, stride=393217) == 3
    assert go(logits=C.c_void_p(0x10002)) == 6 and go(logits=C.c_void_p(0x10001), dtype=1) == 6 and go(token=C.c_void_p(0x10002)) == 6


def test_chunk_attention_refusals(lib):
    n = C.c_size_t()
    assert lib.pt_kernel_chunk_attn_scratch_bytes(0, 1, 1, 128, C.byref(n)) == 1 and lib.pt_kernel_chunk_attn_scratch_bytes(1, 1, 8, 128, None) == 1
    assert lib.pt_kernel_chunk_attn_scratch_bytes(2, 3, 8, 128, C.byref(n)) == 0

    def go(q=FAKE, pool=FAKE, stride=1 << 20, maxp=4, T=2, B=3, M=5, nq=8, nkv=2, dh=128, ps=16, pages=9, out=FAKE, impl=0, scratch=FAKE, sb=n.value, ql=FAKE):
        return lib.pt_kernel_chunk_attn(q, pool, stride, FAKE, maxp, ql, FAKE, T, B, M, nq, nkv, dh, ps, pages, out, impl, scratch, sb, FAKE, None)
    assert go(q=None) == 1 and go(ql=None) == 1 and go(scratch=None) == 1
    for bad in (dict(T=0), dict(B=0), dict(M=0), dict(nq=0), dict(nkv=0), dict(nkv=3), dict(maxp=0), dict(pages=0), dict(ps=12), dict(ps=72), dict(impl=2), dict(stride=-8)):
        assert go(**bad) == 1, bad
    assert go(dh=96) == 3 and go(nq=18) == 3 and go(dh=32) == 3 and go(ps=24) == 3
    assert go(q=C.c_void_p(0x10008)) == 6 and go(out=C.c_void_p(0x10010)) == 6 and go(pool=C.c_void_p(0x10008)) == 6 and go(stride=(1 << 20) + 4) == 6 and go(scratch=C.c_void_p(0x10080)) == 6
    assert go(sb=n.value - 1) == 4


def test_ragged_call_refusals(lib):
    rc, h = make(lib, dtype=pt.PT_BF16)
    c, _ = _cache(lib, h, 6, 16, esz=2)
    n, e = C.c_size_t(), C.c_size_t()
    assert lib.pt_workspace_bytes_ex(h, 40, 4, 16, 0, 0, C.byref(n)) == 0 and lib.pt_extend_workspace_bytes(h, 40, 4, 16, 0, 0, C.byref(e)) == 0
    assert e.value > n.value
    assert lib.pt_extend_workspace_bytes(h, 0, 4, 16, 0, 0, C.byref(e)) == 1 and lib.pt_extend_workspace_bytes(None, 40, 4, 16, 0, 0, C.byref(e)) == 1
    ws = C.c_void_p(0x100000)
    assert lib.pt_extend(h, c, FAKE, 0, 2, None, i32([0, 1]), FAKE, ws, 1 << 30, None) == 1
    assert lib.pt_extend(h, c, FAKE, 0, 2, i32([1, 1]), i32([0, 1]), FAKE, ws, 1 << 30, None) == 10   # weights not bound
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)


def test_generate_sample_refusals(lib):
    sp = pt.pt_sampling()
    rc, h = make(lib, dtype=pt.PT_BF16)
    c, _ = _cache(lib, h, 6, 16, esz=2)
    assert lib.pt_generate_sample(h, c, FAKE, 1, 4, 2, i32([0]), C.byref(sp), FAKE, None, FAKE, 1 << 30, None) == 1      # no random numbers
    assert lib.pt_generate_sample(h, c, FAKE, 1, 4, 2, i32([0]), None, FAKE, None, FAKE, 1 << 30, None) == 1
    lib.pt_kv_cache_free(c)
    lib.pt_model_destroy(h)


def test_python_sampling_arguments_are_checked():
    import torch
    with pytest.raises(ValueError):
        pt.sample(torch.zeros(2, 8), torch.zeros(2))                                                # not on a GPU
