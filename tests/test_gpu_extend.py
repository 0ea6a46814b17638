"""Ragged forward calls (pt_extend) against the oracle and against the uniform calls, and the serving operators together:
one prompt prefilled once, forked, sampled from, speculated tokens checked in ragged calls, pages compacted on the way."""
import numpy as np
import pytest

from oracle import pt_oracle as O
from paper_2602_07306_b200 import inputs as I
from tests import helpers as Hp

pytestmark = pytest.mark.gpu

CASES = {
    "bf16": dict(H=256, nq=4, nkv=2),
    "bf16_dh128": dict(H=512, nq=4, nkv=1),
    "bf16_dh32_ps8": dict(H=128, nq=4, nkv=4, ps=8),
    "f32": dict(H=128, nq=4, nkv=2, dtype="f32", ps=8),
    "e4m3": dict(H=256, nq=2, nkv=1, kv="e4m3"),
    "experts": dict(H=256, nq=4, nkv=4, experts=4, top_k=4),
    "simt_bf16": dict(H=128, nq=2, nkv=2, flags=1),
}


def setup(c, seed=0):
    wl = I.Workload("extend", T=2, L=4, D=2, hidden=c["H"], heads=c["nq"], kv_heads=c["nkv"], ffn=352, dtype=c.get("dtype", "bf16"), mode="prefill", batch=1, seq=8,
                    experts=c.get("experts", 0), top_k=c.get("top_k", 0))
    ws = I.WeightSource(wl, std=0.04, gain_jitter=0.1)
    return wl, ws, Hp.make_model(wl, ws, max_pos=700, flags=c.get("flags", 0))


def draw(wl, rng, *lead):
    x = rng.standard_normal((wl.T,) + lead + (wl.hidden,), dtype=np.float32)
    return I.round_to_bf16(x) if wl.dtype == "bf16" else x


def rounding_floor(wl, ws, history, kv8):
    """Mean relative error over every row of the given sequences (x [T, n, hidden] each) that rounding only what has to be
    bf16 (the contractions' operands and the cache, or the E4M3 codes) leaves inside exact arithmetic.  These weights are
    N(0, 0.04), twice the workloads' 0.02: a projection of a hidden-512 stream has gain 0.04 sqrt(512) = 0.9, the layer
    deltas are as large as the stream, and the floor lies above the workloads' 2e-3 - rows with few keys most of all (an
    average over n cached vectors rounds by 1 / sqrt(n) of one).  So it is measured on the very rows of the run."""
    from tests import bf16_floor as F
    err = size = 0.0
    for x in history:
        h = {}
        for rnd in (False, True):
            cur = [x[t] for t in range(wl.T)]
            for l in range(wl.L):
                cur = [F._layer(cur[t], ws.get(t, l), np.arange(x.shape[1]), wl.heads, wl.kv_heads, wl.head_dim, rnd, kv8) for t in range(wl.T)]
                if (l + 1) % wl.D == 0:
                    cur = [sum(cur)] * wl.T
            h[rnd] = cur[0]
        err += np.abs(h[True] - h[False]).sum()
        size += np.abs(h[False]).sum()
    return err / size


@pytest.mark.parametrize("name", list(CASES))
def test_ragged_calls_follow_the_oracle(name):
    from tests import bf16_floor as F
    c = CASES[name]
    wl, ws, m = setup(c)
    cfg = Hp.oracle_cfg(wl)
    rng = np.random.default_rng(3)
    ps, kv = c.get("ps", 16), c.get("kv", "model")
    pages = 600 // ps + 20
    order = I.free_list_permutation(pages, seed=2)
    cache, oc = m.new_cache(pages, ps, order, kv_dtype=kv), O.PagedKVCache(cfg, pages, ps, order, kv_format=kv)
    tmx, tmean = Hp.tol(wl.dtype)
    history, all_got, all_ref = {}, [], []
    for step, (n, ids) in enumerate([([30, 1, 150], [0, 5, 2]), ([1, 1, 7, 1], [5, 0, 9, 2]), ([5, 133, 1, 3], [2, 9, 0, 5]), ([1], [7])]):
        x = draw(wl, rng, sum(n))
        got = m.extend(cache, Hp.to_dev(m, x), n, ids).cpu().numpy()
        ref = O.pt_extend(cfg, ws, x.astype(np.float64), n, oc, ids)
        assert np.all(np.isfinite(got)) and Hp.rel_errs(got, ref)[0] <= tmx, (name, step, Hp.rel_errs(got, ref))
        assert [cache.length(s) for s in ids] == [oc.length[s] for s in ids]
        all_got.append(got); all_ref.append(ref)
        for e, k, s in zip(np.cumsum(n), n, ids):
            history[s] = np.concatenate([history.get(s, np.zeros((wl.T, 0, wl.hidden))), x[:, e - k:e].astype(np.float64)], 1)
    if wl.dtype == "bf16" and not wl.experts:
        tmean = max(tmean, F.FLOOR_MARGIN * rounding_floor(wl, ws, history.values(), kv == "e4m3"))
    mean = Hp.rel_errs(np.concatenate(all_got), np.concatenate(all_ref))[1]
    assert mean <= tmean, (name, mean, tmean)
    assert m.device_status() == (0, 0)
    m.close()


def test_ragged_and_uniform_calls_agree_and_mix():
    import torch
    wl, ws, m = setup(CASES["bf16"])
    rng = np.random.default_rng(4)
    a, b = m.new_cache(60, 16), m.new_cache(60, 16)
    x = Hp.to_dev(m, draw(wl, rng, 3, 40))
    pa = m.prefill(a, x, [0, 1, 2])
    pb = m.extend(b, x.reshape(wl.T, 120, -1), [40] * 3, [0, 1, 2]).view(3, 40, -1)
    Hp.assert_close(pb.cpu().numpy(), pa.cpu().numpy(), "bf16")
    d = Hp.to_dev(m, draw(wl, rng, 3))
    Hp.assert_close(m.extend(b, d, [1, 1, 1], [0, 1, 2]).cpu().numpy(), m.decode_step(a, d, [0, 1, 2]).cpu().numpy(), "bf16")
    Hp.assert_close(m.decode_step(b, d, [2, 0, 1]).cpu().numpy(), m.extend(a, d, [1, 1, 1], [2, 0, 1]).cpu().numpy(), "bf16")
    s1 = m.extend(a, x[:1, 0, :5].contiguous(), [2, 3], [0, 1])             # one input for all tracks
    s2 = m.extend(b, x[:1, 0, :5].expand(wl.T, 5, -1).contiguous(), [2, 3], [0, 1])
    Hp.assert_close(s1.cpu().numpy(), s2.cpu().numpy(), "bf16")
    assert m.device_status() == (0, 0)
    m.close()


def test_refusals_leave_the_cache_alone():
    import torch
    from paper_2602_07306_b200 import pt
    wl, ws, m = setup(CASES["bf16"])
    rng = np.random.default_rng(5)
    c = m.new_cache(4, 16)
    x = Hp.to_dev(m, draw(wl, rng, 50))
    m.extend(c, x, [50], [0])
    for n, ids, code in (([17], [0], 5), ([1, 1], [0, 0], 1), ([0, 2], [0, 1], 1), ([-1, 3], [0, 1], 1), ([2], [-1], 1), ([660], [0], 1)):
        y = x[:, :1].expand(wl.T, max(1, sum(n)), -1).contiguous()
        with pytest.raises(pt.PtError) as e:
            m.extend(c, y, n, ids)
        assert e.value.code == code, (n, ids)
        assert c.length(0) == 50 and c.length(1) == 0 and c.free_pages() == 0
    with pytest.raises(AssertionError):
        m.extend(c, x, [49], [0])
    m.close()


def test_sampled_answers_of_one_prompt():
    """Prefill once, fork, sample, check speculated tokens raggedly, drop the rejected ones, compact, go on: every hidden state
    follows the oracle fed with the same tokens, every token is the oracle's draw from the library's logits."""
    import torch
    from paper_2602_07306_b200 import pt
    from tests.test_gpu_generate import V, _setup
    wl, ws, m, table, head, gain = _setup(seed=6)
    cfg = Hp.oracle_cfg(wl)
    rng = np.random.default_rng(7)
    pages = 24
    cache, oc = m.new_cache(pages, 16), O.PagedKVCache(cfg, 64, 16)
    emb = lambda tok: np.broadcast_to(I.round_to_bf16(O.embed(table, tok).astype(np.float32)), (wl.T, len(tok), wl.hidden)).astype(np.float64)

    def forward(tok, n, ids):
        t = torch.tensor(tok, dtype=torch.int32, device="cuda")
        h = m.extend(cache, m.embed(t)[None], n, ids)
        ref = O.pt_extend(cfg, ws, emb(np.array(tok)), n, oc, ids)
        Hp.assert_close(h.cpu().numpy(), ref, "bf16")
        return h

    def draw_tokens(h, rows):
        logits, _ = m.lm_head(h[rows].contiguous(), want_tokens=False)
        u = rng.random(len(rows)).astype(np.float32)
        f = dict(temperature=0.8, top_k=40, top_p=0.9, min_p=0.02)
        full = lambda v, dt: torch.full((len(rows),), v, dtype=dt, device="cuda")
        tok, prob = pt.sample(logits, torch.from_numpy(u).cuda(), full(0.8, torch.float32), full(40, torch.int32), full(0.9, torch.float32), full(0.02, torch.float32))
        tok = tok.cpu().tolist()
        for i, x in enumerate(logits.cpu().numpy()):
            want, _, margin = O.sample(x.astype(np.float64), float(u[i]), **{k: v if k == "top_k" else float(np.float32(v)) for k, v in f.items()})
            assert margin < 1e-9 or tok[i] == want
        return tok

    prompt = rng.integers(0, V, 21).tolist()
    h = forward(prompt, [21], [0])
    ids = [0, 1, 2]
    for s in ids[1:]:
        cache.fork(0, s); oc.fork(0, s, 21)
    assert cache.free_pages() == pages - 2
    last = draw_tokens(h, [20, 20, 20])
    for rnd in range(4):
        spec = [int(rng.integers(0, 4)) for _ in ids]                         # so many guessed tokens behind the last one
        rows, n = [], []
        for s, t in zip(spec, last):
            rows += [t] + rng.integers(0, V, s).tolist()
            n.append(1 + s)
        h = forward(rows, n, ids)
        first = np.cumsum([0] + n[:-1])
        last = draw_tokens(h, [int(f) for f in first])                        # no guess is accepted: draw from the first row
        for s, k in zip(ids, n):
            cache.truncate(s, cache.length(s) - (k - 1)); oc.length[s] -= k - 1
        if rnd == 1:
            cache.release(1); oc.release(1)
            cache.fork(2, 1); oc.fork(2, 1, oc.length[2])
            last[1] = last[2]
            cache.compact()
            used = pages - cache.free_pages()
            assert max(p for s in ids for p in cache.block_table(s)) == used - 1
    assert m.device_status() == (0, 0)
    m.close()
