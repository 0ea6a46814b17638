"""What is not a number in a visible place of chunk attention shows in the result, whether or not its keys are split between
blocks: softmax over scores of which one is NaN, or which are all -inf, is NaN in every output of the row and head, and no
other row or head is touched."""
import numpy as np
import pytest

from tests.test_gpu_chunk import call, case, reference

pytestmark = pytest.mark.gpu

# one key; keys of one, two and three tiles of 128 (the second softmax group takes part); enough for all blocks (cut segments)
LAYOUTS = [(1, 4, 2, 128, 16, [1, 2], [1, 40]), (1, 4, 1, 64, 16, [3, 1], [130, 129]), (2, 2, 2, 128, 16, [2, 5], [300, 700]),
           (1, 2, 1, 128, 32, [2, 1], [30000, 9000]), (1, 8, 2, 64, 16, [3], [20001]), (1, 8, 1, 128, 16, [40, 33], [5000, 2600])]


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_nan_query(layout, impl):
    T, nq, nkv, dh, ps, q_len, kv_len = layout
    q, pool, bt = case(*layout, seed=5)
    ref, bound = reference(q, pool, bt, q_len, kv_len, ps)
    row, head = sum(q_len) - 1, nq - 1
    q[:, row, head, 3] = np.nan
    got, status = call(q, pool, bt, q_len, kv_len, ps, impl)
    assert status == [0, 0]
    assert np.all(np.isnan(got[:, row, head])), got[:, row, head, :4]
    got[:, row, head] = ref[:, row, head]
    assert np.all(np.abs(got - ref) <= bound)


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("keys,bad", [(129, 128), (40, 0), (300, 299), (20001, 20000), (20001, 5)])
def test_a_nan_key(keys, bad, impl):
    """The last key alone in its tile (so that nothing else of the tile counts), the first one, ones of cut segments."""
    layout = (1, 2, 2, 128, 16, [1], [keys])
    T, nq, nkv, dh, ps, q_len, kv_len = layout
    q, pool, bt = case(*layout, seed=6)
    ref, bound = reference(q, pool, bt, q_len, kv_len, ps)
    pool[0, bt[0, bad // ps], 0, 1, bad % ps, 7] = np.nan       # K of head 1 only
    got, status = call(q, pool, bt, q_len, kv_len, ps, impl)
    assert status == [0, 0]
    assert np.all(np.isnan(got[0, 0, 1])), got[0, 0, 1, :4]
    assert np.all(np.abs(got - ref)[:, :, 0] <= bound[:, :, 0])


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("keys", [1, 200, 9000])
def test_scores_that_are_all_minus_infinity(keys, impl):
    layout = (1, 2, 2, 64, 16, [1], [keys])
    T, nq, nkv, dh, ps, q_len, kv_len = layout
    q, pool, bt = case(*layout, seed=7)
    ref, bound = reference(q, pool, bt, q_len, kv_len, ps)
    q[:, :, 1] = np.abs(q[:, :, 1]) + np.float32(0.5)
    for j in range(keys):
        pool[0, bt[0, j // ps], 0, 1, j % ps] = -np.inf
    got, status = call(q, pool, bt, q_len, kv_len, ps, impl)
    assert status == [0, 0]
    assert np.all(np.isnan(got[0, 0, 1])), got[0, 0, 1, :4]
    assert np.all(np.abs(got - ref)[:, :, 0] <= bound[:, :, 0])
