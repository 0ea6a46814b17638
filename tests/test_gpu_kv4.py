"""The operators of the 4-bit cache on the GPU, against the oracle's format and the definitions in float64.

Write is compared bit for bit, read value for value (a cached value has six significant bits).  The bound of an element
o = sum p_j v_j of the attention (p the softmax weights, A = sum p_j |v_j|) counts the roundings of the kernel: the result to
bf16 (2^-8 |o|); the weights to fp16 and their products with the scales of V to fp16 (2^-11 A each, and, below fp16's normal
range, 2^-25 of the row's largest weight and of the largest |v| for every key); a score's fp32 sum of dh products (dh 2^-24
sum_i |q_i k_i| scale, twice that for a tensor core that cuts instead of rounding; a q below 2^-24 of its fp16 unit loses
2^-38 of the row's largest); the scale and exp2 in fp32 (2^-24 |s| + 2^-22 each way); fp32 sums over the keys (n 2^-24, for
numerator and denominator).  Slots behind a sequence's last key, unused pages and table entries behind the last page hold NaN
and nonsense: nothing may depend on them."""
import numpy as np
import pytest

from oracle import kv4
from paper_2602_07306_b200 import inputs as I

pytestmark = pytest.mark.gpu


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().bfloat16()


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def crafted(rng, n, dh):
    """Vectors bf16 [n, dh] of every kind."""
    x = rng.standard_normal((n, dh)).astype(np.float32) * np.exp2(rng.integers(-24, 24, (n, 1))).astype(np.float32)
    x[0] = 0
    x[1, :] = -0.0
    x[2] = np.linspace(-6, 6, dh)
    x[3, :8] = [6, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5]
    x[3, 8:] = np.tile([0.125, -0.25], dh)[:dh - 8]
    x[4, 0] = np.nan
    x[5, 33] = np.inf
    x[6, 5], x[6, 40] = 3e38, -3e38
    x[7] = 1e-39
    x[8, :] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6], dh) * 2.0 ** -9 * 1.375        # ties at a scale with all its bits
    x[8, ::32] = 6 * 2.0 ** -9 * 1.375
    x[9] = 6 * 61440.0
    x[10] = 2.0 ** -17 * 6
    x[11] = 2.0 ** -17 * 6.25
    m = 8 + rng.integers(0, 8, (n - 12, 1))
    x[12:] = np.where(rng.random((n - 12, 1)) < 0.3, rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6], (n - 12, dh)) * m * np.exp2(rng.integers(-15, 10, (n - 12, 1))), x[12:])
    return I.round_to_bf16(x)


@pytest.mark.parametrize("T,M,nkv,dh,ps,values", [(1, 1, 1, 128, 16, False), (2, 37, 3, 128, 48, True), (3, 64, 2, 64, 64, True), (2, 300, 1, 64, 16, False), (1, 129, 8, 128, 32, True)])
def test_write(T, M, nkv, dh, ps, values):
    import torch
    from paper_2602_07306_b200 import pt
    rng = np.random.default_rng(M)
    pages = -(-M // ps) + 3
    x = [crafted(rng, max(T * M * nkv, 40), dh)[:T * M * nkv].reshape(T, M, nkv, dh) for _ in range(2)]
    x = [a[:, rng.permutation(M)] for a in x]
    slots = rng.permutation(pages * ps)[:M]
    slots[rng.random(M) < 0.15] = -7
    pool = rng.integers(0, 256, (T, pages, nkv, ps // 16, 17 * dh)).astype(np.uint8)
    want = pool.copy()
    for r in range(M):
        for h in range(nkv):
            if slots[r] >= 0:
                kv4.put(want, slots[r] // ps, h, slots[r] % ps, x[0][:, r, h], x[1][:, r, h])
    got = torch.from_numpy(pool).cuda()
    k, v = (bf(a).view(T, M, nkv * dh) for a in x)
    out = {}
    if values:                                                     # strided rows, as columns of one projection's output
        wide = torch.cat([k, v], -1)
        k, v = wide[..., :nkv * dh], wide[..., nkv * dh:]
        out = dict(k_out=torch.empty((T, M, nkv * dh), dtype=torch.bfloat16, device="cuda"), v_out=torch.empty((T, M, nkv * dh), dtype=torch.bfloat16, device="cuda"))
    status = pt.kernel_kv_write_e2m1(k, v, got, torch.from_numpy(slots).cuda(), nkv=nkv, dh=dh, ps=ps, **out)
    assert status[:2].tolist() == [0, 0]
    assert np.array_equal(got.cpu().numpy(), want)
    if values:
        for a, o in zip(x, (out["k_out"], out["v_out"])):
            np.testing.assert_array_equal(o.float().cpu().numpy().reshape(a.shape).astype(np.float64), kv4.values(*kv4.quantize(a)))


def test_write_in_place_values_and_a_page_outside_the_pool():
    import torch
    from paper_2602_07306_b200 import pt
    rng = np.random.default_rng(3)
    k, v = crafted(rng, 40, 128).reshape(1, 40, 128), crafted(rng, 40, 128).reshape(1, 40, 128)
    slots = rng.permutation(48)[:40]
    slots[17] = 48                                                 # the first slot behind the pool
    slots[19] = 1 << 40
    pool = np.zeros((1, 3, 1, 1, 17 * 128), np.uint8)
    want = pool.copy()
    for r in range(40):
        if slots[r] < 48:
            kv4.put(want, slots[r] // 16, 0, slots[r] % 16, k[:, r], v[:, r])
    got, dk, dv = torch.from_numpy(pool).cuda(), bf(k), bf(v)
    status = pt.kernel_kv_write_e2m1(dk, dv, got, torch.from_numpy(slots).cuda(), nkv=1, dh=128, ps=16, k_out=dk, v_out=dv)
    assert status[:2].tolist() == [8, 24]
    assert np.array_equal(got.cpu().numpy(), want)
    for a, o in ((k, dk), (v, dv)):
        np.testing.assert_array_equal(o.float().cpu().numpy().astype(np.float64), kv4.values(*kv4.quantize(a)))


def cache(T, nkv, dh, ps, kv_len, seed, k_scale=1.0, v_scale=1.0, dead=2, make=None):
    """A pool with poison in every place that no key owns: (bytes uint8, values float64 [T, pages, 2, nkv, ps, dh], block table)."""
    rng = np.random.default_rng(seed)
    B = len(kv_len)
    used = [-(-n // ps) for n in kv_len]
    pages = sum(used) + dead
    order = rng.permutation(pages)
    bt = np.full((B, max(max(used), 1) + 1), -12345, np.int32)
    kc, vc, ks, vs, shift = kv4.places(dh)
    x = rng.standard_normal((2, T, pages, nkv, ps, dh)) * np.array([k_scale, v_scale]).reshape(2, 1, 1, 1, 1, 1)
    at, owned = 0, np.zeros((pages, ps), bool)
    for b in range(B):
        bt[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
        for i in range(used[b]):
            owned[bt[b, i], :kv_len[b] - i * ps] = True
    if make is not None:
        make(x, bt)
    x = I.round_to_bf16(x.astype(np.float32))
    pool = np.zeros((T, pages, nkv, ps // 16, 17 * dh), np.uint8)
    free = ~owned.reshape(1, pages, 1, ps // 16, 16, 1)
    for a, cat, sat in ((x[0], kc, ks), (x[1], vc, vs)):
        code, byte = (z.reshape(T, pages, nkv, ps // 16, 16, -1) for z in kv4.quantize(a))
        code, byte = np.where(free, 15, code), np.where(free, 255, byte)
        pool[..., cat[:, ::2]] = code[..., ::2] | code[..., 1::2] << 4
        pool[..., sat] = byte
    return pool, kv4.get(pool), bt


@pytest.mark.parametrize("T,nkv,dh,ps,ops,kv_len", [
    (1, 1, 128, 16, 16, [1]), (2, 3, 128, 48, 24, [0, 17, 200, 48]), (3, 2, 64, 16, 8, [33, 0, 0, 100]), (1, 8, 64, 64, 64, [640]), (2, 1, 128, 32, 40, [15, 16, 31, 32, 33]),
    (4, 2, 128, 16, 16, [(37 * i) % 61 for i in range(300)])])
def test_read(T, nkv, dh, ps, ops, kv_len):
    import torch
    from paper_2602_07306_b200 import pt
    pool, values, bt = cache(T, nkv, dh, ps, kv_len, seed=len(kv_len) + dh)
    rng = np.random.default_rng(5)
    used = [-(-n // ops) for n in kv_len]
    opages = sum(used) + 2
    order, at = rng.permutation(opages), 0
    obt = np.full((len(kv_len), max(used) + 1), -9, np.int32)
    want = rng.standard_normal((T, opages, 2, nkv, ops, dh)).astype(np.float32)
    want = I.round_to_bf16(want)
    out = bf(want)
    for b, n in enumerate(kv_len):
        obt[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
        for pos in range(n):
            want[:, obt[b, pos // ops], :, :, pos % ops] = values[:, bt[b, pos // ps], :, :, pos % ps]
    _, status = pt.kernel_kv_read_e2m1(torch.from_numpy(pool).cuda(), i32(bt), i32(kv_len), out, i32(obt), nkv=nkv, dh=dh, ps=ps)
    assert status[:2].tolist() == [0, 0]
    np.testing.assert_array_equal(out.float().cpu().numpy(), want)


def test_read_bad_pages_and_lengths_are_reported_and_skipped():
    import torch
    from paper_2602_07306_b200 import pt
    pool, values, bt = cache(1, 2, 64, 16, [40, 20], seed=1)
    dp = torch.from_numpy(pool).cuda()
    obt = np.array([[0, 1, 2], [3, 4, 99]], np.int32)

    def go(bt, lens, obt):
        out = torch.zeros((1, 5, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
        _, st = pt.kernel_kv_read_e2m1(dp, i32(bt), i32(lens), out, i32(obt), nkv=2, dh=64, ps=16)
        return out.float().cpu().numpy()[0], st[:2].tolist()
    good, st = go(bt, [40, 20], obt)
    assert st == [0, 0]
    b2 = bt.copy()
    b2[0, 1] = pool.shape[1]
    got, st = go(b2, [40, 20], obt)
    assert st == [8, 24] and not got[1].any() and np.array_equal(got[[0, 2, 3, 4]], good[[0, 2, 3, 4]])
    o2 = obt.copy()
    o2[1, 0] = 5
    got, st = go(bt, [40, 20], o2)
    assert st == [8, 24] and not got[3].any() and np.array_equal(got[[0, 1, 2, 4]], good[[0, 1, 2, 4]])
    for lens in ([-1, 20], [40, 65], [49, 20]):
        got, st = go(bt[:, :4], lens, obt)
        assert st == [8, 25] and not got.any()


def reference(q, values, bt, q_len, kv_len, ps):
    """(out, bound) float64 [T, rows, nq, dh] on the GPU in double."""
    import torch
    T, _, nq, dh = q.shape
    nkv = values.shape[3]
    G = nq // nkv
    out = torch.zeros((T, sum(q_len), nq, dh), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    dq, dv = torch.from_numpy(q).cuda().double(), torch.from_numpy(values).cuda()
    r = 0
    for b, (S, K) in enumerate(zip(q_len, kv_len)):
        if S:
            pos = torch.arange(K, device="cuda")
            pg = torch.from_numpy(bt[b].astype(np.int64)).cuda()[pos // ps]
            seen = pos[None] <= torch.arange(K - S, K, device="cuda")[:, None]
            for h in range(nkv):
                k, v = (dv[:, pg, i, h, pos % ps][:, None] for i in (0, 1))                      # [T, 1, K, dh]
                a = dq[:, r:r + S, h * G:(h + 1) * G].transpose(1, 2)                            # [T, G, S, dh]
                s = a @ k.transpose(-1, -2) / np.sqrt(dh)
                e = a.abs() @ k.abs().transpose(-1, -2) / np.sqrt(dh)
                tiny = 2.0 ** -38 * a.abs().amax(-1, keepdim=True) * k.abs().sum(-1)[:, :, None] / np.sqrt(dh)
                err = (2 * dh * 2.0 ** -24 * e + tiny + 2.0 ** -23 * s.abs() + 2.0 ** -21).masked_fill(~seen, 0).amax(-1, keepdim=True)
                p = torch.softmax(s.masked_fill(~seen, -np.inf), -1)
                o, A, top = p @ v, p @ v.abs(), v.abs().amax((-1, -2), keepdim=True)
                n = seen.sum(-1)[:, None]
                out[:, r:r + S, h * G:(h + 1) * G] = o.transpose(1, 2)
                lim = 2.0 ** -8 * o.abs() + (A * (2.0 ** -10 + 2.5 * err + 2 * K * 2.0 ** -24) + n * p.amax(-1, keepdim=True) * 2.0 ** -24 * top) * (1 + 2.0 ** -7)
                bound[:, r:r + S, h * G:(h + 1) * G] = lim.transpose(1, 2)
        r += S
    return out.cpu().numpy(), bound.cpu().numpy()


def attend(q, pool, bt, kv_len, q_len, ps, nkv, **kw):
    import torch
    from paper_2602_07306_b200 import pt
    T, M, nq, dh = q.shape
    out, st = pt.kernel_attn_e2m1(bf(q).view(T, M, nq * dh), torch.from_numpy(pool).cuda(), i32(bt), i32(kv_len), None if q_len is None else i32(q_len),
                                  nq=nq, nkv=nkv, dh=dh, ps=ps, **kw)
    return out.view(T, M, nq, dh), st[:2].tolist()


def queries(T, rows, nq, dh, seed, scale=1.0):
    return I.round_to_bf16(np.random.default_rng(seed + 99).standard_normal((T, rows, nq, dh)).astype(np.float32) * scale)


def check(T, nq, nkv, dh, ps, q_len, kv_len, seed=0, scale=1.0, make=None, extra=0, k_scale=1.0, v_scale=1.0):
    pool, values, bt = cache(T, nkv, dh, ps, kv_len, seed, k_scale=k_scale, v_scale=v_scale, make=make)
    ql = [1] * len(kv_len) if q_len is None else q_len
    q = queries(T, sum(ql) + extra, nq, dh, seed, scale)
    want, bound = reference(q, values, bt, ql, kv_len, ps)
    import torch
    filled = torch.full((T, q.shape[1], nq * dh), 7.0, dtype=torch.bfloat16, device="cuda")
    got, st = attend(q, pool, bt, kv_len, q_len, ps, nkv, out=filled)
    assert st == [0, 0]
    got = got.float().cpu().numpy().astype(np.float64)
    assert (got[:, sum(ql):] == 7).all()                           # rows behind the last sequence stay
    d = np.abs(got[:, :sum(ql)] - want)
    assert np.isfinite(d).all() and (d <= bound).all(), (float(d.max()), float((d / np.maximum(bound, 1e-300)).max()))
    again, _ = attend(q, pool, bt, kv_len, q_len, ps, nkv)
    assert np.array_equal(again.float().cpu().numpy()[:, :sum(ql)], got[:, :sum(ql)])      # the same bits


@pytest.mark.parametrize("T,nq,nkv,dh,ps,q_len,kv_len", [
    (1, 1, 1, 128, 16, None, [1]),
    (1, 1, 1, 64, 16, None, [2, 1, 16, 17]),
    (4, 8, 8, 64, 16, None, [301]),
    (2, 8, 1, 128, 64, None, [5000]),
    (2, 16, 4, 128, 16, None, [1, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 500]),
    (3, 6, 2, 128, 48, None, [47, 48, 49, 95, 96, 97, 1000]),
    (1, 10, 2, 64, 32, None, [2000, 3, 700]),
    (1, 8, 8, 128, 16, [4], [301]),
    (2, 8, 8, 128, 16, [0, 8, 3, 0, 1, 5, 0], [5, 900, 3, 0, 17, 40, 33]),
    (1, 16, 2, 128, 32, [5, 5], [700, 5]),
    (2, 12, 4, 64, 16, [1, 33, 2], [200, 100, 2]),
    (1, 8, 1, 128, 16, [70], [70]),
    (1, 5, 1, 64, 48, [7, 129], [3000, 1500]),
    (2, 16, 4, 128, 16, None, [200 + (977 * i) % 700 for i in range(60)]),
    (1, 2, 1, 128, 16, [i % 4 for i in range(700)], [i % 4 + (31 * i) % 70 for i in range(700)]),
])
def test_attention(T, nq, nkv, dh, ps, q_len, kv_len):
    check(T, nq, nkv, dh, ps, q_len, kv_len, seed=sum(kv_len), extra=2 if q_len else 0)


@pytest.mark.parametrize("scale,k_scale,v_scale", [(8.0, 4.0, 1.0), (2.0 ** -20, 1.0, 2.0 ** -13), (2.0 ** 40, 2.0 ** -40, 1.0), (1.0, 1.0, 2.0 ** 14), (2.0 ** -30, 2.0 ** 12, 2.0 ** -17)])
def test_attention_magnitudes(scale, k_scale, v_scale):
    """Peaked scores, flat ones, and K, V and q at the ends of the formats' ranges."""
    check(1, 8, 2, 128, 16, None, [900, 40], seed=1, scale=scale, k_scale=k_scale, v_scale=v_scale)


def test_attention_scores_that_climb_and_v_that_grows():
    def make(x, bt):
        n = 1200
        pos = np.arange(n)
        pg, sl = bt[0, pos // 16], pos % 16
        u = queries(1, 1, 4, 128, 5)[0, 0]                          # the queries of the call below
        x[0, 0, pg, 0, sl] = 0.3 * x[0, 0, pg, 0, sl] + (pos / n)[:, None] * 3.0 * u[0]
        x[0, 0, pg, 1, sl] += (pos >= 700)[:, None] * 2.5 * u[2]
        x[1, 0, pg, 0, sl] *= np.exp2(np.floor(pos * 24 / n) - 12)[:, None]
        x[1, 0, pg, 1, sl] *= np.exp2(8 - np.floor(pos * 16 / n))[:, None]
    check(1, 4, 2, 128, 16, None, [1200], seed=5, make=make)


def test_attention_nan_and_infinities():
    """A group that is not finite reads as NaN: in K the rows that see it are NaN, in V the columns of the group."""
    import torch
    def make(x, bt):
        x[0, 0, bt[0, 2], 0, 3, 5] = np.nan                        # key 35 of sequence 0, head 0
        x[1, 0, bt[0, 4], 1, 1, 70] = np.inf                       # value 65, head 1, group 2
        x[0, 0, bt[1, 0], 1, 15, 0] = np.inf                       # key 15 of sequence 1, head 1: seen by its last row alone
    pool, values, bt = cache(1, 2, 128, 16, [100, 16], 8, make=make)
    q = queries(1, 5, 4, 128, 8)
    got, st = attend(q, pool, bt, [100, 16], [1, 4], 16, 2)
    got = got.float().cpu().numpy()[0]
    assert st == [0, 0]
    assert np.isnan(got[0, :2]).all() and np.isnan(got[0, 2:, 64:96]).all() and np.isfinite(got[0, 2:, :64]).all() and np.isfinite(got[0, 2:, 96:]).all()
    assert np.isfinite(got[1:4]).all() and np.isfinite(got[4, :2]).all() and np.isnan(got[4, 2:]).all()
    q[0, 0, 3, 9] = np.inf                                         # and a query that is not finite: its own head alone
    got2, _ = attend(q, pool, bt, [100, 16], [1, 4], 16, 2)
    got2 = got2.float().cpu().numpy()[0]
    assert np.isnan(got2[0, 3]).all() and np.array_equal(got2[0, 2], got[0, 2], equal_nan=True) and np.array_equal(got2[1:4], got[1:4])


@pytest.mark.parametrize("nq,nkv,dh,S,K", [(2, 2, 128, 8, 60), (2, 2, 64, 5, 33), (8, 2, 128, 4, 70), (8, 2, 64, 4, 200), (16, 2, 128, 3, 50), (10, 2, 64, 4, 31), (4, 1, 128, 40, 90),
                                          (1, 1, 64, 70, 70), (2, 1, 128, 3, 3000)])
def test_attention_values_that_are_not_finite_stay_with_the_rows_that_see_them(nq, nkv, dh, S, K):
    """The same call with zeros in their groups gives the other rows, and the other columns, bit for bit."""
    G, mid = nq // nkv, K - S + S // 2
    def make(fill):
        def at(x, bt):
            for key, head, group, value in ((mid, 0, 1, fill and np.nan), (mid, nkv - 1, 0, fill and -np.inf), (K - 1, nkv - 1, dh // 32 - 1, fill and np.inf)):
                x[1, 0, bt[0, key // 16], head, key % 16, 32 * group:32 * group + 32] = 0
                x[1, 0, bt[0, key // 16], head, key % 16, 32 * group + 7] = value
        return at
    q = queries(1, S, nq, dh, 8)
    got = []
    for fill in (0, 1):
        pool, _, bt = cache(1, nkv, dh, 16, [K], 8, make=make(fill))
        out, st = attend(q, pool, bt, [K], [S], 16, nkv)
        assert st == [0, 0]
        got.append(out.float().cpu().numpy()[0])
    want = got[0]
    assert np.isfinite(want).all()
    want[S // 2:, :G, 32:64] = np.nan
    want[S // 2:, nq - G:, :32] = np.nan
    want[S - 1:, nq - G:, dh - 32:] = np.nan
    assert np.array_equal(got[1], want, equal_nan=True)


def test_attention_bad_pages_and_lengths_are_reported():
    pool, values, bt = cache(2, 2, 128, 16, [60, 40, 20], 4)
    q = queries(2, 3, 4, 128, 4)
    good, st = attend(q, pool, bt, [60, 40, 20], None, 16, 2)
    assert st == [0, 0]
    for page in (-1, pool.shape[1]):
        b2 = bt.copy()
        b2[1, 2] = page
        got, st = attend(q, pool, b2, [60, 40, 20], None, 16, 2)
        assert st == [8, 24]
        for r in (0, 2):
            assert np.array_equal(got[:, r].float().cpu().numpy(), good[:, r].float().cpu().numpy())
    import torch
    for ql, kl in (([1, 1, 1], [60, 81, 20]), ([1, 1, 2], [60, 40, 20]), ([1, -1, 1], [60, 40, 20]), ([1, 1, 1], [60, 0, 20])):
        out = torch.full((2, 3, 512), 7.0, dtype=torch.bfloat16, device="cuda")
        got, st = attend(q, pool, bt, kl, ql, 16, 2, out=out)
        assert st == [8, 25] and (got == 7).all()


def test_attention_replayed_with_other_lengths():
    """A captured call reads its lengths and tables when it runs."""
    import torch
    from paper_2602_07306_b200 import pt
    pool, values, bt = cache(2, 2, 128, 16, [900, 500], 6)
    q = queries(2, 6, 8, 128, 6)
    dev = dict(pool=torch.from_numpy(pool).cuda(), bt=i32(bt), kv=i32([30, 20]), ql=i32([1, 1]), q=bf(q).view(2, 6, 1024))
    out, status = torch.zeros_like(dev["q"]), torch.zeros(16, dtype=torch.int32, device="cuda")
    scratch = pt.attn_e2m1_scratch(2, 8, 2, 128)
    call = lambda: pt.kernel_attn_e2m1(dev["q"], dev["pool"], dev["bt"], dev["kv"], dev["ql"], nq=8, nkv=2, dh=128, ps=16, out=out, scratch=scratch, status=status)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
    for ql, kl in (([1, 1], [900, 500]), ([4, 2], [900, 37]), ([0, 3], [0, 500])):
        dev["kv"].copy_(i32(kl)), dev["ql"].copy_(i32(ql))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        want, _ = attend(q, pool, bt, kl, ql, 16, 2)
        assert status[:2].tolist() == [0, 0]
        assert np.array_equal(out.view(2, 6, 8, 128).float().cpu().numpy()[:, :sum(ql)], want.float().cpu().numpy()[:, :sum(ql)])


def test_write_read_and_attend_together():
    """Tokens written step by step; the attention from the codes equals the library's bf16 attention over what is read back,
    to the roundings of both (2^-8 of the result each, 2^-8 and 2^-10 of the weights)."""
    import torch
    from paper_2602_07306_b200 import pt
    T, B, nq, nkv, dh, ps = 2, 3, 8, 2, 128, 32
    rng = np.random.default_rng(2)
    pages, maxp = 24, 8
    bt = rng.permutation(pages)[:B * maxp].reshape(B, maxp).astype(np.int32)
    pool = torch.full((T, pages, nkv, ps // 16, 17 * dh), 255, dtype=torch.uint8, device="cuda")
    lens = [0] * B
    shape = dict(nkv=nkv, dh=dh, ps=ps)
    for new in ([100, 31, 7], [1, 1, 1], [0, 3, 120], [1, 1, 1], [5, 2, 4]):
        slots = np.concatenate([bt[b, p // ps] * ps + p % ps for b in range(B) for p in [np.arange(lens[b], lens[b] + new[b])]])
        k, v, q = (bf(rng.standard_normal((T, len(slots), h * dh))) for h in (nkv, nkv, nq))
        lens = [a + b for a, b in zip(lens, new)]
        assert pt.kernel_kv_write_e2m1(k, v, pool, torch.from_numpy(slots).cuda(), **shape)[0] == 0
        out, st = pt.kernel_attn_e2m1(q, pool, i32(bt), i32(lens), i32(new), nq=nq, **shape)
        obt = np.arange(B * 16, dtype=np.int32).reshape(B, 16)
        flat = torch.full((T, B * 16, 2, nkv, 16, dh), float("nan"), dtype=torch.bfloat16, device="cuda")
        _, st2 = pt.kernel_kv_read_e2m1(pool, i32(bt), i32(lens), flat, i32(obt), **shape)
        want, st3 = pt.kernel_chunk_attn(q, flat, i32(obt), i32(new), i32(lens), nq=nq, nkv=nkv, dh=dh, ps=16)
        assert [s[0].item() for s in (st, st2, st3)] == [0, 0, 0]
        top = torch.nan_to_num(flat.float()).abs().amax()
        d = (out.float() - want.float()).abs()
        assert (d <= 2.0 ** -7 * want.float().abs() + (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -12) * top).all(), d.max()


@pytest.mark.parametrize("T,nq,nkv,dh,q_len,kv_len", [(2, 4, 2, 128, None, [301, 40, 17]), (1, 8, 8, 64, [3, 0, 1], [90, 5, 33]), (1, 8, 2, 128, [9, 20], [64, 300])])
def test_attention_of_short_sequences_under_a_wide_table(T, nq, nkv, dh, q_len, kv_len):
    """Few short segments take a thread block each where the table says that they are short, and are cut up where it does not."""
    import torch
    pool, values, bt = cache(T, nkv, dh, 16, kv_len, 11)
    ql = [1] * len(kv_len) if q_len is None else q_len
    q = queries(T, sum(ql), nq, dh, 11)
    want, bound = reference(q, values, bt, ql, kv_len, 16)
    for columns in (bt.shape[1], 500):
        wide = np.full((len(kv_len), columns), -5, np.int32)
        wide[:, :bt.shape[1]] = bt
        got, st = attend(q, pool, wide, kv_len, q_len, 16, nkv)
        d = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
        assert st == [0, 0] and np.isfinite(d).all() and (d <= bound).all(), columns


def test_calls_without_work():
    """Sequences without new tokens, or without keys, leave everything as it was."""
    import torch
    from paper_2602_07306_b200 import pt
    pool, values, bt = cache(1, 2, 64, 16, [30, 10], 12)
    q = queries(1, 3, 4, 64, 12)
    out = torch.full((1, 3, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    for ql, kl in (([0, 0], [30, 10]), ([0, 0], [0, 0])):
        got, st = attend(q, pool, bt, kl, ql, 16, 2, out=out)
        assert st == [0, 0] and (got == 7).all()
    dp = torch.from_numpy(pool).cuda()
    k = torch.randn((1, 5, 128), device="cuda").bfloat16()
    st = pt.kernel_kv_write_e2m1(k, k, dp, torch.full((5,), -1, dtype=torch.int64, device="cuda"), nkv=2, dh=64, ps=16)
    assert st[0] == 0 and np.array_equal(dp.cpu().numpy(), pool)
    e = torch.empty((1, 0, 128), dtype=torch.bfloat16, device="cuda")
    assert pt.kernel_kv_write_e2m1(e, e, dp, torch.empty(0, dtype=torch.int64, device="cuda"), nkv=2, dh=64, ps=16)[0] == 0


def test_pools_beyond_32_bit_offsets():
    """Pages more than 2^32 bytes into a track's slab, and a second track behind them."""
    import torch
    from paper_2602_07306_b200 import pt
    nkv, dh, ps, n = 8, 128, 64, 150
    pages = (1 << 32) // (nkv * (ps // 16) * 17 * dh) + 40
    pool = torch.empty((2, pages, nkv, ps // 16, 17 * dh), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(0)
    bt = np.array([[pages - 1, pages - 30, pages - 7]], np.int32)
    pool[:, torch.from_numpy(bt[0]).long().cuda()] = 255
    k, v = (I.round_to_bf16(rng.standard_normal((2, n, nkv, dh)).astype(np.float32)) for _ in range(2))
    pos = np.arange(n)
    slots = bt[0, pos // ps].astype(np.int64) * ps + pos % ps
    shape = dict(nkv=nkv, dh=dh, ps=ps)
    st = pt.kernel_kv_write_e2m1(bf(k).view(2, n, -1), bf(v).view(2, n, -1), pool, torch.from_numpy(slots).cuda(), **shape)
    assert st[0] == 0
    near = np.zeros((2, 3, nkv, ps // 16, 17 * dh), np.uint8)
    near[:] = 255
    for p in range(n):
        for h in range(nkv):
            kv4.put(near, p // ps, h, p % ps, k[:, p, h], v[:, p, h])
    assert np.array_equal(pool[:, torch.from_numpy(bt[0]).long().cuda()].cpu().numpy(), near)
    values = kv4.get(near)
    out = torch.zeros((2, 10, 2, nkv, 16, dh), dtype=torch.bfloat16, device="cuda")
    _, st = pt.kernel_kv_read_e2m1(pool, i32(bt), i32([n]), out, i32([np.arange(10)]), **shape)
    assert st[0] == 0
    flat = np.moveaxis(out.float().cpu().numpy(), 4, 2).reshape(2, 160, 2, nkv, dh)[:, :n]
    np.testing.assert_array_equal(flat, np.moveaxis(values, 4, 2).reshape(2, 3 * ps, 2, nkv, dh)[:, :n])
    q = queries(2, 2, nkv, dh, 3)
    want, bound = reference(q, values, np.array([[0, 1, 2]], np.int32), [2], [n], ps)
    got, st = pt.kernel_attn_e2m1(bf(q).view(2, 2, -1), pool, i32(bt), i32([n]), i32([2]), nq=nkv, **shape)
    d = np.abs(got.view(2, 2, nkv, dh).float().cpu().numpy().astype(np.float64) - want)
    assert st[0] == 0 and (d <= bound).all()


def test_two_streams_at_once():
    """Calls on two streams, each with a scratch of its own, give what they give alone."""
    import torch
    from paper_2602_07306_b200 import pt
    cases = []
    for seed in (1, 2):
        pool, values, bt = cache(2, 4, 128, 16, [700 + 100 * seed, 900, 33], seed)
        cases.append(dict(q=bf(queries(2, 3, 16, 128, seed)).view(2, 3, -1), pool_l=torch.from_numpy(pool).cuda(), block_table=i32(bt),
                          kv_len=i32([700 + 100 * seed, 900, 33]), nq=16, nkv=4, dh=128, ps=16, scratch=pt.attn_e2m1_scratch(2, 16, 4, 128)))
    alone = [pt.kernel_attn_e2m1(**c)[0].clone() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.empty_like(c["q"]) for _ in range(20)] for c in cases]
    for i in range(20):
        for s, c, o in zip(streams, cases, outs):
            with torch.cuda.stream(s):
                pt.kernel_attn_e2m1(**c, out=o[i])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, x) for x in o)


def test_a_captured_step_replayed():
    """Write, attention and read back of one decode step in a graph: replayed with other tokens, slots and lengths."""
    import torch
    from paper_2602_07306_b200 import pt
    T, B, nq, nkv, dh, ps = 2, 3, 8, 2, 128, 16
    rng = np.random.default_rng(4)
    bt = rng.permutation(30)[:B * 8].reshape(B, 8).astype(np.int32)
    shape = dict(nkv=nkv, dh=dh, ps=ps)
    pool = torch.zeros((T, 30, nkv, 1, 17 * dh), dtype=torch.uint8, device="cuda")
    first = np.concatenate([bt[b, np.arange(60) // ps] * ps + np.arange(60) % ps for b in range(B)]).astype(np.int64)
    k0, v0 = (bf(rng.standard_normal((T, B * 60, nkv * dh))) for _ in range(2))
    pt.kernel_kv_write_e2m1(k0, v0, pool, torch.from_numpy(first).cuda(), **shape)
    k, v, q = (torch.zeros((T, B, h * dh), dtype=torch.bfloat16, device="cuda") for h in (nkv, nkv, nq))
    slots, lens, table = torch.full((B,), -1, dtype=torch.int64, device="cuda"), i32([60] * B), i32(bt)
    out, flat = torch.zeros_like(q), torch.zeros((T, B * 8, 2, nkv, 16, dh), dtype=torch.bfloat16, device="cuda")
    obt, scratch, status = i32(np.arange(B * 8).reshape(B, 8)), pt.attn_e2m1_scratch(T, nq, nkv, dh), torch.zeros(16, dtype=torch.int32, device="cuda")

    def step():
        pt.kernel_kv_write_e2m1(k, v, pool, slots, status=status, **shape)
        pt.kernel_attn_e2m1(q, pool, table, lens, nq=nq, out=out, scratch=scratch, status=status, **shape)
        pt.kernel_kv_read_e2m1(pool, table, lens, flat, obt, status=status, **shape)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for n in (61, 62, 63):
        for x in (k, v, q):
            x.copy_(bf(rng.standard_normal(x.shape)))
        slots.copy_(torch.from_numpy((bt[:, (n - 1) // ps] * ps + (n - 1) % ps).astype(np.int64)))
        lens.copy_(i32([n] * B))
        g.replay()
        torch.cuda.synchronize()
        got, copy = out.clone(), flat.clone()
        other = torch.empty_like(out)
        pt.kernel_attn_e2m1(q, pool, table, lens, nq=nq, out=other, **shape)
        want, _ = pt.kernel_chunk_attn(q, copy, obt, i32([1] * B), lens, nq=nq, nkv=nkv, dh=dh, ps=16)
        assert status[0] == 0 and torch.equal(got, other)
        top = copy.float().abs().amax()
        assert ((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -12) * top).all()
        values = kv4.get(pool.cpu().numpy())
        for b in range(B):
            last = values[:, bt[b, (n - 1) // ps], :, :, (n - 1) % ps]
            np.testing.assert_array_equal(last[:, 0].reshape(T, -1), kv4.values(*kv4.quantize(k[:, b].float().cpu().numpy().reshape(T, nkv, dh))).reshape(T, -1))
            np.testing.assert_array_equal(copy.float().cpu().numpy()[:, b * 8 + (n - 1) // 16, :, :, (n - 1) % 16], last)
