"""Pins of the oracle's serving pieces (sampling filters, forked sequences, ragged batches) to hand-worked values, closed
forms and independent formulations."""
import numpy as np
import pytest
import torch

from oracle import pt_oracle as O
from paper_2602_07306_b200 import inputs as I


def test_filters_keep_the_hand_worked_sets():
    x = np.log([4.0, 2.0, 2.0, 1.0, 1.0])                    # weights 1, 1/2, 1/2, 1/4, 1/4 of the largest
    keep = lambda **f: O.sample_kept(x, **f)[0].tolist()
    assert keep() == [0, 1, 2, 3, 4]
    assert keep(top_k=2) == [0, 1]                           # the tie goes to the lower index
    assert keep(top_k=5) == keep(top_k=0) == keep(top_k=-1) == keep(top_k=9) == [0, 1, 2, 3, 4]
    assert keep(top_p=0.39) == [0] and keep(top_p=0.41) == [0, 1] and keep(top_p=0.61) == [0, 1, 2] and keep(top_p=0.81) == [0, 1, 2, 3]
    assert keep(top_p=0.0) == [0]
    assert keep(top_k=3, top_p=0.55) == [0, 1]               # top-p counts against what top-k left: 4 + 2 of 8
    assert keep(min_p=0.4) == [0, 1, 2] and keep(min_p=0.6) == [0] and keep(min_p=5.0) == [0]
    assert keep(temperature=0.5, min_p=0.3) == [0]           # weights 1, 1/4, 1/16 at half the temperature
    assert keep(temperature=0.0) == keep(temperature=float("nan")) == [0]
    assert O.sample_kept(np.array([-np.inf, np.nan]))[0].tolist() == []
    assert O.sample_kept(np.array([1.0, np.inf, np.inf]))[0].tolist() == [0, 1, 2] and O.sample_kept(np.array([1.0, np.inf, np.inf]))[1].tolist() == [0, 1, 1]


def test_the_draw_inverts_the_softmax():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(37) * 2
    t = 0.7
    p = torch.softmax(torch.from_numpy(x / t), 0).numpy()
    edges = np.concatenate([[0.0], np.cumsum(p)])
    for i in range(37):                                      # the middle of every token's interval, and just inside its ends
        for u in (0.5 * (edges[i] + edges[i + 1]), edges[i] + 1e-9, edges[i + 1] - 1e-9):
            tok, pr, _ = O.sample(x, u, temperature=t)
            assert tok == i and abs(pr - p[i]) < 1e-12
    assert O.sample(x, -1.0)[0] == O.sample(x, float("nan"))[0] == 0 and O.sample(x, 2.0)[0] == 36


def _cfg():
    wl = I.Workload("pins", T=2, L=2, D=1, hidden=64, heads=2, kv_heads=1, ffn=96, dtype="f32", mode="prefill", batch=1, seq=4)
    return wl, I.WeightSource(wl, std=0.2), O.PTConfig(T=2, D=1, L=2, hidden=64, heads=2, kv_heads=1, ffn=96)


def test_a_ragged_batch_equals_single_sequences_and_uniform_batches():
    wl, ws, cfg = _cfg()
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 9, 64))
    a, b = O.PagedKVCache(cfg, 8, 8), O.PagedKVCache(cfg, 8, 8)
    got = O.pt_extend(cfg, ws, x, [4, 1, 4], a, [0, 1, 2])
    uni = O.pt_prefill(cfg, ws, np.stack([x[:, :4], x[:, 5:]], 1), b, [0, 2])
    np.testing.assert_allclose(got[:4], uni[0], atol=1e-12)
    np.testing.assert_allclose(got[5:], uni[1], atol=1e-12)
    np.testing.assert_allclose(got[4:5], O.pt_prefill(cfg, ws, x[:, None, 4:5], b, [1])[0], atol=1e-12)
    assert [a.length[s] for s in (0, 1, 2)] == [4, 1, 4]


@pytest.mark.parametrize("n", [0, 3, 8, 11])
def test_a_forked_sequence_continues_like_one_prefilled_with_the_prefix(n):
    wl, ws, cfg = _cfg()
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((2, 1, 11, 64)), rng.standard_normal((2, 1, 5, 64))
    c = O.PagedKVCache(cfg, 12, 8)
    O.pt_prefill(cfg, ws, x, c, [0])
    c.fork(0, 1, n)
    got = O.pt_prefill(cfg, ws, y, c, [1])
    O.pt_prefill(cfg, ws, y, c, [0])                         # the source goes its own way
    ref = O.PagedKVCache(cfg, 12, 8)
    want = O.pt_prefill(cfg, ws, np.concatenate([x[:, :, :n], y], 2), ref, [7])[:, n:]
    np.testing.assert_allclose(got, want, atol=1e-12)
