"""Sampling on the GPU against the oracle's float64 statement of it: every token must be the oracle's, wherever no decision
(a step of the cumulative distribution against u, the reach of top-p, min-p's threshold) is closer than the arithmetic can
tell apart.

How close is that?  A weight is held to 2^-45 of the largest (rounded to a multiple of 2^-44) and computed in double, so a
sum of n weights is off by at most n 2^-45 (1 + small): relative to the kept sum Z, n 2^-45 / Z.  Both sides of a decision
carry it: 2 n 2^-45 / Z + 1e-13 for the double arithmetic of either side.  Inputs are drawn so that hardly any row is closer
(the share skipped is checked)."""
import numpy as np
import pytest

from oracle import pt_oracle as O

pytestmark = pytest.mark.gpu

# probability: rounded to fp32 once (2^-24), the kept sum off by n 2^-45
PROB_REL = lambda n: 2.0 ** -24 + n * 2.0 ** -45 + 1e-12


def dev(a, dt=None):
    import torch
    t = torch.from_numpy(np.array(a)).cuda()
    return t if dt is None else t.to(dt)


def run(x, u, bf16=False, pad=0, **f):
    """x float32 [n, V] (already representable), filters as arrays or scalars -> (tokens, probs)"""
    import torch
    from paper_2602_07306_b200 import pt
    n, V = x.shape
    full = torch.full((n, V + pad), 1e9, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")     # the padding must not be read as logits
    full[:, :V] = dev(x)
    arr = lambda a, dt: None if a is None else dev(np.broadcast_to(np.asarray(a, dt), (n,)))
    tok, prob = pt.sample(full[:, :V], dev(np.asarray(u, np.float32)), arr(f.get("temperature"), np.float32), arr(f.get("top_k"), np.int32),
                          arr(f.get("top_p"), np.float32), arr(f.get("min_p"), np.float32))
    torch.cuda.synchronize()
    return tok.cpu().numpy(), prob.cpu().numpy()


def check(x, u, bf16=False, pad=0, most_skipped=0.02, **f):
    n, V = x.shape
    tok, prob = run(x, u, bf16, pad, **f)
    skipped = 0
    for r in range(n):
        g = {}
        for k, dt in (("temperature", np.float32), ("top_k", np.int64), ("top_p", np.float32), ("min_p", np.float32)):
            if f.get(k) is not None:
                g[k] = np.broadcast_to(np.asarray(f[k], dt), (n,))[r].astype(np.float64 if dt is np.float32 else np.int64)
        want, p, margin = O.sample(x[r].astype(np.float64), float(np.float32(u[r])), **g)
        Z = O.sample_kept(x[r].astype(np.float64), **g)[1].sum() or 1.0
        if margin < 2 * V * 2.0 ** -45 / Z + 1e-13:
            skipped += 1
            continue
        assert tok[r] == want, (r, tok[r], want, margin, g)
        assert abs(float(prob[r]) - p) <= PROB_REL(V) * p, (r, prob[r], p)         # (in double: fp32 would round the difference)
    assert skipped <= most_skipped * n, skipped


SHAPES = [(1, 1), (2, 2), (4, 3), (3, 33), (5, 1000), (2, 16384), (3, 16385), (2, 40001), (2, 65537), (2, 131073), (1, 200001), (1, 393216)]


@pytest.mark.parametrize("n,V", SHAPES)
@pytest.mark.parametrize("mode", ["plain", "k", "p", "m", "all"])
def test_matches_the_oracle(n, V, mode):
    rng = np.random.default_rng(V + len(mode))
    x = (rng.standard_normal((n, V)) * 2.5).astype(np.float32)
    f = {"plain": dict(temperature=0.9), "k": dict(temperature=1.1, top_k=max(1, V // 7)), "p": dict(top_p=0.9), "m": dict(temperature=1.3, min_p=0.03),
         "all": dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.01)}[mode]
    check(x, rng.random(n), pad=V % 3, **f)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("scale", [0.05, 1.0, 4.0, 40.0])
def test_rows_with_their_own_settings(bf16, scale):
    import torch
    n, V = 48, 20011
    rng = np.random.default_rng(int(scale * 100))
    x = (rng.standard_normal((n, V)) * scale).astype(np.float32)
    if bf16:                                                  # many exact ties
        x = torch.from_numpy(x).bfloat16().float().numpy()
    x[rng.random((n, V)) < 0.3] = -np.inf
    pick = lambda a: rng.choice(a, n)
    check(x, rng.random(n), bf16=bf16, pad=5, temperature=pick([0.0, 0.2, 1.0, 1.7]), top_k=pick([0, 1, 2, 37, 5000, 20010]),
          top_p=pick([1.0, 0.3, 0.9, 0.999]), min_p=pick([0.0, 0.01, 0.5]))


@pytest.mark.parametrize("n,V", [(3, 50001), (40, 70003), (300, 4099), (2, 300007)])
@pytest.mark.parametrize("f", [dict(top_k=5000, top_p=0.9), dict(top_k=3000, temperature=1.4), dict(top_p=0.5), dict(top_p=0.9999, min_p=1e-4), dict(top_p=1e-7), dict(top_k=700, min_p=0.02),
                               dict(temperature=3.0), dict(top_p=1 - 2.0 ** -24)], ids=str)
def test_long_selections_in_few_and_in_many_rows(n, V, f):
    """A large top-k with and without top-p behind it, reaches close to 0 and 1, both ways of holding a row, odd strides."""
    rng = np.random.default_rng(n + V)
    x = (rng.standard_normal((n, V)) * 2).astype(np.float32)
    x[:, rng.integers(0, V, V // 5)] = -np.inf
    check(x, rng.random(n), pad=3, most_skipped=0.05, **f)


def test_every_kept_token_is_reached_and_no_other():
    """One row, a dense grid of u: the tokens drawn are exactly the kept ones, each on its share of the grid."""
    V, n = 300, 4000
    rng = np.random.default_rng(3)
    x = np.repeat((rng.standard_normal((1, V)) * 1.5).astype(np.float32), n, 0)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    for f in (dict(top_k=9), dict(top_p=0.7), dict(min_p=0.2), dict(temperature=2.0, top_k=40, top_p=0.8, min_p=0.1)):
        tok, prob = run(x, u, **f)
        ids, w, _ = O.sample_kept(x[0].astype(np.float64), **{k: float(np.float32(v)) if k != "top_k" else v for k, v in f.items()})
        assert set(tok.tolist()) <= set(ids.tolist()) and np.all(np.diff(tok) >= 0)
        share = np.bincount(tok, minlength=V)[ids] / n
        assert np.abs(share - w / w.sum()).max() <= 1.0 / n + 1e-6     # an interval of length l holds between l n - 1 and l n + 1 grid points
        check(x, u, most_skipped=0.01, **f)


def test_ties_take_the_lowest_indices():
    V = 30000
    x = np.zeros((6, V), np.float32)                          # all equal: the first k of them
    x[1, ::2] = -1.0
    x[2, 100:] = -0.0                                         # -0 equals +0
    u = np.array([0.999999, 0.999999, 0.999999, 0.0, 0.25, 0.5], np.float32)
    tok, prob = run(x, u, top_k=1000)
    assert tok[0] == 999 and tok[1] == 1999 and tok[2] == 999 and tok[3] == 0 and tok[4] == 250 and tok[5] == 500
    assert np.all(prob == np.float32(1e-3))
    tok, _ = run(x[:1], u[:1], top_p=0.5)                     # the shortest prefix that holds half of the weight
    assert tok[0] == V // 2 - 1
    tok, _ = run(x[:1], u[:1], top_k=64, top_p=0.25)          # dyadic: sixteen of sixty-four exactly
    assert tok[0] == 15
    for V2, k in ((1500, 1000), (2048, 1024), (2000, 700)):  # lists of nothing but ties
        y = np.zeros((3, V2), np.float32)
        y[1, 100:] = -0.5
        tok, prob = run(y, np.array([0.5, 0.999999, 0.0], np.float32), top_k=k)
        assert tok[0] == k // 2 and tok[1] == k - 1 and tok[2] == 0, (V2, k, tok)
    # ties that straddle several blocks' slices, with larger values in front and behind
    y = np.full((1, 120000), -3.0, np.float32)
    y[0, 70000:90000] = 1.0
    y[0, 5] = y[0, 119999] = 2.0
    tok, _ = run(np.repeat(y, 3, 0), np.array([0.0, 0.5, 0.9999999], np.float32), top_k=10002)
    assert tok[0] == 5 and tok[2] == 119999 and 70000 <= tok[1] < 80000


def test_masked_rows_and_special_values():
    V = 5000
    inf, nan = np.inf, np.nan
    low = np.float32(-3.4028235e38)
    x = np.zeros((10, V), np.float32)
    x[0] = -inf                                               # nothing left
    x[1] = nan
    x[2] = -inf; x[2, 4321] = -7.0                            # one token left
    x[3] = low                                                # a mask of the type's lowest value everywhere: all equal
    x[4] = low; x[4, 17] = 3.0
    x[5, :] = 1.0; x[5, 9] = inf; x[5, 77] = inf              # +inf shares the weight
    x[6] = nan; x[6, 3] = 0.5; x[6, 4] = -inf
    x[7] = 3.4028235e38; x[7, 11] = -3.4028235e38
    x[8] = np.linspace(-1e-38, 1e-38, V)                      # subnormal differences
    x[9, 1:] = -30.0                                          # weights of 1e-13
    u = np.array([0.3, 0.3, 0.3, 0.5, 0.9, 0.75, 0.2, 0.5, 0.5, 0.9], np.float32)
    for f in (dict(), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=4000, top_p=0.5, min_p=0.1), dict(temperature=0.0)):
        tok, prob = run(x, u, **f)
        assert tok[0] == 0 and prob[0] == 0 and tok[1] == 0 and prob[1] == 0
        assert tok[2] == 4321 and prob[2] == 1
        assert tok[4] == 17 and tok[6] == 3
        greedy = f.get("temperature") == 0.0
        assert tok[5] == (9 if greedy or f.get("top_p") is not None and f["top_p"] <= 0.5 else 77), (f, tok[5])
        if not f:
            assert tok[3] == V // 2 and tok[7] in (V // 2, V // 2 + 1) and tok[8] in (V // 2 - 1, V // 2, V // 2 + 1)
        assert tok[9] == 0
        assert np.all(np.isfinite(prob)) and np.all((tok >= 0) & (tok < V))


def test_rows_at_the_ends_of_the_number_range():
    """Rows of the type's lowest value with and without -inf among it, logits whose steps are coarse next to the temperature."""
    inf, low, V = np.inf, np.float32(-3.4028235e38), 4000
    for bf16 in (False, True):
        lo = np.float32(-3.3895314e38) if bf16 else low
        x = np.full((4, V), lo, np.float32)
        x[1, ::2] = -inf
        x[2, :] = -inf; x[2, [7, 9]] = lo
        x[3, 5] = 0.0
        tok, prob = run(x, np.array([0.5, 0.5, 0.75, 0.9], np.float32), bf16=bf16)
        assert tok.tolist() == [V // 2, V // 2 + 1, 9, 5], tok
        assert np.allclose(prob, [1 / V, 2 / V, 0.5, 1.0], rtol=1e-6, atol=0)
    big = np.float32(1e8)                                     # steps of 8
    x = np.repeat((big - 8 * np.arange(V)[::-1]).astype(np.float32)[None], 6, 0)
    check(x, np.linspace(0.05, 0.95, 6), temperature=4.0)
    check(x, np.linspace(0.05, 0.95, 6), temperature=np.array([1e-6, 0.3, 1.0, 100.0, 1e5, 1e9]), top_k=900)
    check(x, np.linspace(0.05, 0.95, 6), temperature=np.array([1e-6, 0.3, 1.0, 100.0, 1e5, 1e9]), top_p=0.8)


def test_edges_of_u_and_of_the_settings():
    V = 777
    rng = np.random.default_rng(8)
    x = np.repeat(rng.standard_normal((1, V)).astype(np.float32), 9, 0)
    u = np.array([0.0, -1.0, np.nan, 1.0, 2.0, np.inf, 1 - 2.0 ** -24, 2.0 ** -149, -np.inf], np.float32)
    tok, _ = run(x, u)
    assert tok[0] == tok[1] == tok[2] == tok[8] == 0 and np.all(tok[3:7] == V - 1) and tok[7] == 0
    best = int(np.argmax(x[0]))
    n = 9
    for f in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=np.nan), dict(temperature=np.inf), dict(top_p=0.0), dict(top_p=-1.0), dict(min_p=1.0), dict(min_p=7.0),
              dict(top_k=1), dict(temperature=1e-30), dict(temperature=1e-42)):
        tok, prob = run(x, u, **f)
        assert np.all(tok == best) and np.all(prob == 1), f
    base, _ = run(x, rng.random(n))
    u = rng.random(n)
    want, _ = run(x, u)
    for f in (dict(top_k=0), dict(top_k=-5), dict(top_k=V), dict(top_k=2 ** 31 - 1), dict(top_p=1.0), dict(top_p=np.nan), dict(top_p=9.0), dict(min_p=0.0), dict(min_p=np.nan), dict(min_p=-1.0)):
        tok, _ = run(x, u, **f)
        assert np.array_equal(tok, want), f
    tok, _ = run(x, u, temperature=1e38)                      # as good as uniform
    assert np.array_equal(tok, np.minimum((np.float32(u).astype(np.float64) * V).astype(np.int64), V - 1))


def test_a_row_does_not_depend_on_its_batch_and_calls_repeat():
    rng = np.random.default_rng(11)
    x = (rng.standard_normal((70, 33000)) * 2).astype(np.float32)
    u = rng.random(70)
    f = dict(temperature=1.2, top_k=500, top_p=0.9, min_p=0.001)
    tok, prob = run(x, u, **f)
    again, prob2 = run(x, u, **f)
    assert np.array_equal(tok, again) and np.array_equal(prob, prob2)
    for r in (0, 33, 69):
        t1, p1 = run(x[r:r + 1], u[r:r + 1], **f)
        assert t1[0] == tok[r] and p1[0] == prob[r]


@pytest.mark.parametrize("f", [dict(), dict(top_k=40), dict(top_k=700, top_p=0.8), dict(top_k=5000), dict(top_p=0.9), dict(top_k=9000, top_p=0.6, min_p=1e-5), dict(min_p=0.01), dict(temperature=0.0)], ids=str)
def test_every_way_of_taking_a_row_gives_the_same(f):
    """1 to 150 rows at once: clusters that hold their slices, clusters that stream over them, a block a row.  The sums are whole
    numbers, so the draws and their probabilities are equal bit for bit."""
    rng = np.random.default_rng(12)
    V = 70001
    x = (rng.standard_normal((150, V)) * 2).astype(np.float32)
    x[1] = -np.inf
    x[2] = 0.25                                               # all equal
    x[3, 5:] = np.nan
    x[4, 100:] = -3.4028235e38
    x[5, 69000] = np.inf
    x[6] = np.floor(x[6])                                     # few values, thousands of times each
    x[7] *= 20
    u = rng.random(150)
    u[:3] = [0.0, 0.5, 0.999]
    tok, prob = run(x, u, pad=2, **f)
    for n in (1, 9, 30, 40, 70, 100):
        t, p = run(x[:n], u[:n], pad=2, **f)
        assert np.array_equal(t, tok[:n]) and np.array_equal(p, prob[:n]), n


def test_a_captured_call_replays_on_new_logits_and_on_another_stream():
    import torch
    from paper_2602_07306_b200 import pt
    rng = np.random.default_rng(12)
    logits, u = dev((rng.standard_normal((5, 9000)) * 2).astype(np.float32)), dev(rng.random(5).astype(np.float32))
    tok, prob = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
    top_p = torch.full((5,), 0.9, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        pt.sample(logits, u, top_p=top_p, out=tok, prob=prob)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            pt.sample(logits, u, top_p=top_p, out=tok, prob=prob)
    st.synchronize()
    for _ in range(3):
        x, uu = (rng.standard_normal((5, 9000)) * 2).astype(np.float32), rng.random(5).astype(np.float32)
        logits.copy_(dev(x)); u.copy_(dev(uu))
        g.replay()
        torch.cuda.synchronize()
        want, _ = run(x, uu, top_p=0.9)
        assert np.array_equal(tok.cpu().numpy(), want)


def test_generate_with_sampling_draws_from_its_own_logits():
    import torch
    from paper_2602_07306_b200 import pt
    from tests.test_gpu_generate import V, _setup
    wl, ws, model, table, head, gain = _setup(seed=4)
    rng = np.random.default_rng(5)
    B, S, n_new = 3, 9, 7
    prompt = dev(rng.integers(0, V, (B, S)).astype(np.int32))
    u = dev(rng.random((n_new, B)).astype(np.float32))
    t, p = torch.tensor([0.7, 1.0, 0.0], device="cuda"), torch.tensor([0.9, 0.5, 1.0], device="cuda")
    k = torch.tensor([20, 0, 0], dtype=torch.int32, device="cuda")
    prob = torch.zeros(B, n_new, device="cuda")
    cache = model.new_cache(8, 16)
    tok, logits = model.generate(cache, prompt, n_new, [0, 1, 2], want_logits=True, u=u, temperature=t, top_k=k, top_p=p, prob=prob)
    torch.cuda.synchronize()
    assert model.device_status() == (0, 0)
    for i in range(n_new):
        want, wp = pt.sample(logits[:, i].contiguous(), u[i].contiguous(), t, k, p)
        assert torch.equal(tok[:, i], want) and torch.equal(prob[:, i], wp)
    assert torch.equal(tok[2], logits[2].argmax(-1).int())    # temperature 0: the greedy choice
    with pytest.raises(ValueError):
        model.generate(cache, prompt, n_new, [4, 5, 6], u=u[:, :2].contiguous())
    model.close()


def test_python_arguments_are_checked():
    import torch
    from paper_2602_07306_b200 import pt
    x, u = torch.zeros(2, 8, device="cuda"), torch.zeros(2, device="cuda")
    for bad in (dict(temperature=torch.ones(3, device="cuda")), dict(top_k=torch.ones(2, device="cuda")), dict(top_p=torch.ones(2)),
                dict(min_p=torch.ones(4, device="cuda")[::2]), dict(out=torch.zeros(2, device="cuda")), dict(prob=torch.zeros(2, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            pt.sample(x, u, **bad)
    for a, b in ((x.half(), u), (x[:, ::2], u), (x[0], u), (x, u.double()), (x, None), (x, u[:1])):
        with pytest.raises((ValueError, AttributeError)):
            pt.sample(a, b)
