"""How a call on a cache attends, as pt_call_context tells it before the call (no GPU work)."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07306_b200 import pt
from tests.test_host_api import lib                           # noqa: F401  (a fixture)

FAKE = C.c_void_p(0x10000)
PASS, COPY = {8: 1.0, 16: 1.6, 24: 2.0}, 6.0                  # times of a pass over the keys by its rows, and of the copy


def cost(lens, n_new, G):
    """{rows a pass: time}, time of the copy."""
    return {r: t * sum(k * -(-n * G // r) for k, n in zip(lens, n_new)) for r, t in PASS.items()}, COPY * sum(lens)


def ask(lib, cache, n_new, ids=None):
    n, i = (np.array(a, np.int32) for a in (n_new, range(len(n_new)) if ids is None else ids))
    ctx, rows = C.c_int64(-1), C.c_int32(-1)
    st = lib.pt_call_context(cache, len(n), n.ctypes.data_as(C.POINTER(C.c_int32)), i.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(ctx), C.byref(rows))
    return st, ctx.value, rows.value


@pytest.fixture
def model(lib):
    made = []

    def make(heads, kv, kv_dtype, max_pos=40000):
        cfg, h, c, n = pt.pt_config(2, 2, 4, 128 * heads, heads, kv, 352, 10000.0, 1e-6, pt.PT_BF16, 0, max_pos, 0, 0, 0), C.c_void_p(), C.c_void_p(), C.c_size_t()
        assert lib.pt_model_create(C.byref(cfg), C.byref(h)) == 0
        assert lib.pt_kv_cache_bytes_ex(h, 4, 16, kv_dtype, C.byref(n)) == 0
        assert lib.pt_kv_cache_alloc_ex(h, 4, 16, kv_dtype, FAKE, n.value, C.byref(c)) == 0
        made.append((h, c))
        return c
    yield make
    for h, c in made:
        lib.pt_kv_cache_free(c)
        lib.pt_model_destroy(h)


def test_uneven_calls_are_planned_by_rows_and_keys(lib, model):
    """One sequence of 64 rows among many of one: the mean of the rows says nothing about the keys that are read."""
    c = model(2, 2, pt.PT_KV_E2M1)
    assert ask(lib, c, [64] + [1] * 31) == (0, 0, 24)         # a pass of 8 rows would read its keys eight times
    assert ask(lib, c, [1] * 32) == (0, 0, 8)
    assert ask(lib, c, [16] * 3) == (0, 0, 16)
    assert ask(lib, c, [150, 1, 1]) == (0, 160 + 16 + 16, 0)  # a prompt: the copy
    assert ask(lib, c, [72]) == (0, 0, 24) and ask(lib, c, [73]) == (0, 80, 0)


@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 1), (8, 1), (6, 2)])
def test_the_cheapest_way_is_taken(lib, model, heads, kv):
    c, rng, ways = model(heads, kv, pt.PT_KV_E2M1), np.random.default_rng(heads), set()
    for _ in range(400):
        n = np.exp(rng.uniform(0, np.log(120), rng.integers(1, 12))).astype(int)
        passes, copy = cost(n, n, heads // kv)
        st, ctx, rows = ask(lib, c, n)
        assert st == 0 and (rows > 0) == (ctx == 0)
        if rows:
            assert passes[rows] <= min(min(passes.values()), copy) * (1 + 1e-12)
        else:
            assert ctx == sum((int(a) + 15) // 16 * 16 for a in n) and min(passes.values()) > copy * (1 - 1e-12)
        ways.add(rows)
    assert ways == {0, 8, 16, 24}


def test_other_formats_and_refusals(lib, model):
    assert ask(lib, model(2, 2, pt.PT_KV_MODEL), [5, 100]) == (0, 0, 0)
    c = model(2, 2, pt.PT_KV_E4M3)
    assert ask(lib, c, [5, 100]) == (0, 16 + 112, 0)
    for n in ([0], [3, -1], [40001], []):
        assert ask(lib, c, n)[0] == 1
    one, ctx = np.array([1], np.int32), C.c_int64()
    p = one.ctypes.data_as(C.POINTER(C.c_int32))
    for a in ((None, 1, p, p, C.byref(ctx)), (c, 1, None, p, C.byref(ctx)), (c, 1, p, None, C.byref(ctx)), (c, 1, p, p, None)):
        assert lib.pt_call_context(*a, None) == 1
    assert lib.pt_call_context(c, 1, p, p, C.byref(ctx), None) == 0 and ctx.value == 16
