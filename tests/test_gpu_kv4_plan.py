"""Calls on a 4-bit cache whose sequences differ much in rows and keys, against the oracle, with the way that pt_call_context tells."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07306_b200 import pt
from tests import helpers as Hp
from tests.test_gpu_kv4_model import Run, draw, four, setup    # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def rows_a_pass(r, n, ids):
    a, b = (np.array(x, np.int32) for x in (n, ids))
    ctx, rows, p = C.c_int64(), C.c_int32(), C.POINTER(C.c_int32)
    pt.check(pt.lib().pt_call_context(r.c.h, len(n), a.ctypes.data_as(p), b.ctypes.data_as(p), C.byref(ctx), C.byref(rows)))
    return rows.value, ctx.value


@pytest.mark.parametrize("H,nq,nkv", [(256, 2, 2), (256, 4, 2), (512, 4, 1)])
def test_uneven_calls_follow_the_oracle(four, H, nq, nkv):     # noqa: F811
    wl, ws, m = setup(H, nq, nkv)
    rng = np.random.default_rng(3)
    r = Run(wl, ws, m, 16, 120)
    G = nq // nkv
    r.prefill(draw(wl, rng, 1, 700), [0])
    r.prefill(draw(wl, rng, 6, 3), [1, 2, 3, 4, 5, 6])
    # many rows over many keys beside single tokens over few: passes of 24 rows
    n, ids = [1, 1, 64 // G, 1, 1, 1, 1], [1, 2, 0, 3, 4, 5, 6]
    assert rows_a_pass(r, n, ids) == (24, 0)
    r.extend(draw(wl, rng, sum(n)), n, ids)
    # and the other way around: the long context has one row
    n, ids = [48 // G, 1, 48 // G], [1, 0, 2]
    assert rows_a_pass(r, n, ids) == (8, 0)
    r.extend(draw(wl, rng, sum(n)), n, ids)
    n, ids = [1, 120, 1], [1, 0, 2]                             # a chunk: the copy of all
    assert rows_a_pass(r, n, ids)[0] == 0 and rows_a_pass(r, n, ids)[1] == sum((r.c.length(s) + k + 15) // 16 * 16 for s, k in zip(ids, n))
    r.extend(draw(wl, rng, sum(n)), n, ids)
    r.check(f"uneven calls, heads {nq}/{nkv}")
    m.close()


def test_calls_straight_to_the_codes_reserve_no_copy():
    """Speculated tokens and short prompts on long contexts: the workspaces have no room for the bf16 copy that is not made."""
    wl, ws, m = setup(256, 2, 1)
    rng, n = np.random.default_rng(4), pt._SZ()
    c = m.new_cache(200, 16, kv_dtype="e2m1")
    m.prefill(c, Hp.to_dev(m, draw(wl, rng, 3, 800)), [0, 1, 2])
    assert c.call_context([800] * 3, [3, 4, 5]) == 2400 and c.call_context([5, 1, 1], [0, 1, 2]) == 0
    m.ws, m.ws_key = None, (0, 0, 0)                           # as a server that has another model object for its decode steps
    m.extend(c, Hp.to_dev(m, draw(wl, rng, 7)), [5, 1, 1], [0, 1, 2])
    m.prefill(c, Hp.to_dev(m, draw(wl, rng, 3, 2)), [0, 1, 2])
    pt.check(pt.lib().pt_extend_workspace_bytes(m.h, 7, 3, 16, pt.PT_KV_E2M1, 0, C.byref(n)))
    assert m.ext_ws.numel() == n.value and m.ext_key[4] == 0
    pt.check(pt.lib().pt_workspace_bytes_ex(m.h, 6, 3, 16, pt.PT_KV_E2M1, 0, C.byref(n)))
    assert m.ws.numel() == n.value and m.ws_key[4] == 0
    assert m.device_status() == (0, 0)
    m.close()
