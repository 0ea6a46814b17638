"""Reaches of top-p next to 1 over rows of a few equal logits, exactly.

Such rows are where the weights' rounding to multiples of 2^-44 of the largest shows: every one of thousands of equal logits is
rounded the same way, and what top-p leaves out (k 2^-24 of the sum) is only a few thousand of them.  The expected token is found
in whole numbers from the definition: w_i = round(2^44 exp(x_i - max)), the shortest prefix of (logit descending, index ascending)
with sum >= ceil(p whole), the lowest index whose cumulative kept weight exceeds floor(u Z).  Logits are drawn so that no weight is
near a half, so the whole numbers do not depend on the exponential's last bits: the tokens have to be equal.  Probabilities: one
rounding to fp32 (2^-24) and double arithmetic (1e-12)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

INV_BIN = 4095 / 31.5                                         # the kernel's bins per nat at temperature 1


def weight(x):
    w = math.exp(float(np.float32(x))) * 2.0 ** 44
    return round(w), abs(w - math.floor(w) - 0.5)


def tail_value(rng, units):
    """fp32 logit close to a bin's edge whose weight is about `units`, a tenth or more from a half"""
    b = round((44 * math.log(2) - math.log(units)) * INV_BIN)
    while True:
        x = np.float32(-(b + rng.choice([-3e-2, -1e-2, -1e-3, 1e-3, 1e-2, 3e-2, 0.3])) / INV_BIN)
        if weight(x)[1] > 0.1:
            return x
        b -= 1


def row(rng, V, k, spread):
    """A maximum of 0, equal logits that weigh about k 2^20 together (what p = 1 - k 2^-24 leaves out), with or without a few larger ones"""
    x = np.full(V, -np.inf, np.float32)
    # many equal logits go through a list of up to 2048 or, beyond that, through exact histograms: both, with small and large weights
    want = int(min(V - 200, rng.choice([300, 1400, 2040, 2500, V // 2, V - 200])))
    t = tail_value(rng, min(max(k * 2.0 ** 20 / want, 0.7), 1e6))
    n = min(V - 200, max(1, round(k * 2 ** 20 / weight(t)[0]) + int(rng.integers(-2, 3)))) if weight(t)[0] else V - 200
    at = rng.permutation(V)
    x[at[:n]] = t
    if spread:                                                # larger weights in front of the equal ones
        t2 = np.float32(-20.0)
        while weight(t2)[1] < 0.1:
            t2 = np.nextafter(t2, np.float32(0))
        x[at[n:n + 100]] = t2
    x[at[-1]] = 0.0
    return x


def expected(x, k, u):
    vals, inv = np.unique(x, return_inverse=True)
    ws = np.array([0 if v == -np.inf else weight(v)[0] for v in vals], np.int64)
    w = ws[inv.reshape(-1)]
    order = np.argsort(-x, kind="stable")
    whole = int(w.sum())
    need = -(-whole * (2 ** 24 - k) // 2 ** 24)
    kept = int(np.searchsorted(np.cumsum(w[order]), need)) + 1
    keep = np.zeros(len(x), bool)
    keep[order[:kept]] = True
    cum = np.cumsum(np.where(keep, w, 0))
    Z = int(cum[-1])
    target = Z * int(float(np.float32(u)) * 2 ** 24) // 2 ** 24          # u is a multiple of 2^-24 here
    tok = int(np.searchsorted(cum, target, side="right"))
    return tok, math.exp(float(x[tok])) / (Z * 2.0 ** -44)


# clusters that hold a row (8, 4, 2 blocks and one), clusters that stream it, a block per row
@pytest.mark.parametrize("n,V", [(3, 24001), (16, 24001), (64, 24001), (300, 24001), (5, 290101), (64, 128003), (2, 393216), (40, 3001), (320, 3001)])
def test_reaches_next_to_one_with_equal_tails(n, V):
    import torch
    from paper_2602_07306_b200 import pt
    rng = np.random.default_rng(n * 1000003 + V)
    x = np.empty((n, V), np.float32)
    ks = np.arange(n) % 16 + 1
    ks[4::5] = rng.choice([64, 300, 2000], len(ks[4::5]))
    for i in range(n):
        x[i] = row(rng, V, int(ks[i]), i % 3 == 2)
    u = (1.0 - rng.choice([1, 1, 2, 3, 9, 2 ** 23, 2 ** 24], n) * 2.0 ** -24).astype(np.float32)
    p = (1.0 - ks * 2.0 ** -24).astype(np.float32)
    d = lambda a: torch.from_numpy(a).cuda()
    tok = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((n,), -7.0, dtype=torch.float32, device="cuda")
    pt.sample(d(x), d(u), top_p=d(p), out=tok, prob=prob)
    torch.cuda.synchronize()
    tok, prob = tok.cpu().numpy(), prob.cpu().numpy().astype(np.float64)
    want = [expected(x[i], int(ks[i]), u[i]) for i in range(n)]
    wrong = [(i, int(ks[i]), int(tok[i]), want[i][0]) for i in range(n) if tok[i] != want[i][0]]
    assert not wrong, (len(wrong), wrong[:5])
    for i in range(n):
        assert abs(prob[i] - want[i][1]) <= (2.0 ** -24 + 1e-12) * want[i][1], (i, prob[i], want[i])


def test_the_two_rows_found_by_reading():
    """1440 logits of 728.36 units, and 290000 of 3.55 behind a hundred larger ones: the cut lies in another bin than unrounded weights say."""
    import torch
    from paper_2602_07306_b200 import pt
    a = np.full(1441, -23.907684, np.float32); a[7] = 0.0
    b = np.full(290101, -29.2313, np.float32); b[5] = 0.0; b[100:200] = -20.0
    for x in (a, b):
        for u in (0.0, 0.5, 1 - 2.0 ** -24):
            # a call before it that leaves other thresholds behind in the blocks' shared memory
            pt.sample(torch.full((300, len(x)), 3.0, device="cuda"), torch.zeros(300, device="cuda"), top_p=torch.full((300,), 1e-6, device="cuda"))
            for n in (1, 300):
                tok = torch.full((n,), -7, dtype=torch.int32, device="cuda")
                d = lambda v: torch.full((n,), v, dtype=torch.float32, device="cuda")
                pt.sample(torch.from_numpy(np.repeat(x[None], n, 0)).cuda(), d(u), top_p=d(1 - 2.0 ** -24), out=tok)
                assert set(tok.tolist()) == {expected(x, 1, u)[0]}, (len(x), u, n, tok[:4].tolist(), expected(x, 1, u))
