"""Ragged calls and the generate loop of a model that holds part of a larger stack's tracks: the all-reduce hook gets the
workspace of the call that runs, whichever of the model's workspaces that is."""
import numpy as np
import pytest

from paper_2602_07306_b200 import inputs as I
from tests import helpers as Hp

pytestmark = pytest.mark.gpu


def workload():
    wl = I.Workload("tp_extend", T=4, L=4, D=2, hidden=256, heads=4, kv_heads=2, ffn=352, dtype="bf16", mode="prefill", batch=1, seq=8)
    return wl, I.WeightSource(wl, gain_jitter=0.1)


@pytest.mark.parametrize("warm", [False, True])
def test_a_ragged_call_reduces_once_per_track_block(warm):
    import torch
    wl, ws = workload()
    rng = np.random.default_rng(1)
    steps = [([30, 1, 70], [0, 1, 2]), ([1, 4, 1], [2, 1, 0])]
    xs = [I.round_to_bf16(rng.standard_normal((wl.T, sum(n), wl.hidden), dtype=np.float32)) for n, _ in steps]
    outs, sizes = [], []
    for hooked in (False, True):
        m = Hp.make_model(wl, ws, max_pos=512)
        cache = m.new_cache(30, 16)
        if warm:                                              # the other workspace exists already
            m.prefill(cache, Hp.to_dev(m, xs[0][:, None, :5]), [9])
        if hooked:
            m.set_track_group(wl.T, lambda t: sizes.append(t.numel()))
        outs.append([m.extend(cache, Hp.to_dev(m, x), n, ids).cpu().numpy() for x, (n, ids) in zip(xs, steps)])
        assert m.device_status() == (0, 0)
        m.close()
    assert sizes == [sum(n) * wl.hidden for n, _ in steps for _ in range(wl.L // wl.D)]
    for a, b in zip(*outs):                                   # the two schedules add the partial sums of squares in a different order
        mx, mean = Hp.rel_errs(a, b)
        assert mx <= 1e-2 and mean <= 2.5e-3, (mx, mean)


def test_generate_under_a_track_group():
    import torch
    wl, ws = workload()
    rng = np.random.default_rng(2)
    V, B, S, new = 208, 2, 6, 3
    table, head = (I.round_to_bf16(rng.standard_normal((V, wl.hidden), dtype=np.float32)) for _ in range(2))
    m = Hp.make_model(wl, ws, max_pos=512)
    m.load_lm(table, head, np.ones(wl.hidden, np.float32))
    calls = []
    m.set_track_group(wl.T, lambda t: calls.append(t.numel()))
    prompt = torch.from_numpy(rng.integers(0, V, (B, S)).astype(np.int32)).cuda()
    m.generate(m.new_cache(8, 16), prompt, new, [0, 1], u=torch.rand((new, B), device="cuda"))
    torch.cuda.synchronize()
    blocks = wl.L // wl.D
    assert calls == [B * S * wl.hidden] * blocks + [B * wl.hidden] * (blocks * (new - 1))
    m.close()
