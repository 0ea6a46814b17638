"""Attention of a ragged chunk over the paged cache: both kernels against the definition in float64, element by element.

The bound of an element o = sum p_j v_j (p the softmax weights, A = sum p_j |v_j|), from the roundings either kernel makes:
the result to bf16 (2^-8 |o|), the probabilities to bf16 in front of P V (2^-8 A; their sum is taken unrounded), a score's
fp32 sum of dh products (dh 2^-24 sum_i |q_i k_i| scale =: e, which moves a probability by a factor exp(2e) at most), the
scale and exp2 in fp32 (2^-24 |s| + 2^-22 each way, s in powers of two), and fp32 sums over the keys and key ranges (n 2^-24,
for the numerator and for the denominator).  Unused slots of a sequence's last page, unused pages and table entries behind the
last page hold NaN and nonsense: nothing may depend on them."""
import numpy as np
import pytest

from paper_2602_07306_b200 import inputs as I

pytestmark = pytest.mark.gpu


def case(T, nq, nkv, dh, ps, q_len, kv_len, seed=0, scale=1.0, extra_rows=0, dead=3):
    """Random q and cache with poison in every place that no key owns.  Returns numpy (bf16-representable float32)."""
    rng = np.random.default_rng(seed)
    B = len(q_len)
    used = [-(-n // ps) for n in kv_len]
    pages = sum(used) + dead
    maxp = max(max(used), 1) + 1
    order = rng.permutation(pages)
    bt = np.full((B, maxp), -12345, np.int32)
    pool = np.full((T, pages, 2, nkv, ps, dh), np.nan, np.float32)
    at = 0
    for b in range(B):
        bt[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
        for i in range(used[b]):
            n = min(ps, kv_len[b] - i * ps)
            pool[:, bt[b, i], :, :, :n] = I.round_to_bf16(rng.standard_normal((T, 2, nkv, n, dh), dtype=np.float32))
    M = sum(q_len) + extra_rows
    q = I.round_to_bf16(rng.standard_normal((T, M, nq, dh), dtype=np.float32) * scale)
    return q, pool, bt


def reference(q, pool, bt, q_len, kv_len, ps):
    """(out, bound) float64 [T, rows, nq, dh], on the GPU in double for the large cases"""
    import torch
    T, M, nq, dh = q.shape
    nkv = pool.shape[3]
    G = nq // nkv
    out = torch.zeros((T, sum(q_len), nq, dh), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    dq, dp = torch.from_numpy(q).cuda(), torch.from_numpy(pool).cuda()
    r = 0
    for b, (S, K) in enumerate(zip(q_len, kv_len)):
        if S:
            pg = torch.from_numpy(bt[b, : -(-K // ps)].astype(np.int64)).cuda()
            seen = torch.arange(K, device="cuda")[None] <= torch.arange(K - S, K, device="cuda")[:, None]
            for t in range(T):
                kv = dp[t, pg].double()
                for h in range(nkv):
                    k, v = (kv[:, i, h].reshape(-1, dh)[:K] for i in (0, 1))
                    for j in range(h * G, h * G + G):
                        a = dq[t, r:r + S, j].double()
                        s = (a @ k.T) / np.sqrt(dh)
                        e = (a.abs() @ k.abs().T) / np.sqrt(dh)
                        err = (dh * 2.0 ** -24 * e + 2.0 ** -23 * s.abs() + 2.0 ** -21).masked_fill(~seen, 0).amax(-1, keepdim=True)
                        p = torch.softmax(s.masked_fill(~seen, -np.inf), -1)
                        o, A = p @ v, p @ v.abs()
                        out[t, r:r + S, j] = o
                        bound[t, r:r + S, j] = 2.0 ** -8 * o.abs() + A * (2.0 ** -8 + 2.5 * err + 2 * K * 2.0 ** -24) * (1 + 2.0 ** -7)
        r += S
    return out.cpu().numpy(), bound.cpu().numpy()


def call(q, pool, bt, q_len, kv_len, ps, impl=None, **kw):
    import torch
    from paper_2602_07306_b200 import pt
    T, M, nq, dh = q.shape
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    out = torch.full((T, M, nq * dh), 5.0, dtype=torch.bfloat16, device="cuda")
    got, status = pt.kernel_chunk_attn(d(q.reshape(T, M, nq * dh)).bfloat16(), d(pool).bfloat16(), d(bt), d(np.asarray(q_len, np.int32)), d(np.asarray(kv_len, np.int32)),
                                       nq=nq, nkv=pool.shape[3], dh=dh, ps=ps, out=out, impl=impl, **kw)
    torch.cuda.synchronize()
    return got.float().cpu().numpy().astype(np.float64).reshape(T, M, nq, dh), status[:2].tolist()


def check(T, nq, nkv, dh, ps, q_len, kv_len, impl, **kw):
    q, pool, bt = case(T, nq, nkv, dh, ps, q_len, kv_len, **kw)
    got, status = call(q, pool, bt, q_len, kv_len, ps, impl)
    assert status == [0, 0]
    n = sum(q_len)
    ref, bound = reference(q, pool, bt, q_len, kv_len, ps)
    err = np.abs(got[:, :n] - ref)
    assert np.all(np.isfinite(got)) and np.all(err <= bound), (float((err / np.maximum(bound, 1e-300)).max()), np.argwhere(err > bound)[:3].tolist())
    assert np.all(got[:, n:] == 5.0), "rows behind the last sequence were written"


SHAPES = [
    # T, nq, nkv, dh, ps, q_len, kv_len
    (1, 1, 1, 128, 16, [1], [1]),                                  # one token, one key
    (1, 4, 4, 64, 16, [3], [3]),
    (2, 8, 8, 128, 16, [4, 0, 1, 7], [4, 0, 130, 257]),            # an empty sequence, chunks at the start and behind a context
    (2, 8, 2, 128, 16, [5, 5, 5], [128, 129, 127]),                # key counts around a tile
    (1, 6, 2, 64, 32, [1, 40, 2], [300, 41, 1000]),                # three query heads per KV head
    (1, 5, 1, 128, 48, [50, 1], [700, 49]),                        # five
    (2, 14, 2, 64, 64, [19, 37], [64, 2049]),                      # seven
    (1, 8, 1, 128, 16, [33, 16, 17], [33, 500, 4000]),             # eight: chunks of one row tile and one more
    (3, 3, 3, 128, 16, [128, 129, 127, 256, 257], [128, 400, 1000, 256, 600]),
    (1, 2, 1, 64, 16, [300], [3333]),
    (1, 16, 4, 128, 16, [1] * 23 + [200] + [1] * 9, [17 * i + 1 for i in range(23)] + [1500] + [900 - i for i in range(9)]),
    (4, 4, 4, 64, 16, [2], [9000]),                                # a long context for few rows
    (1, 2, 2, 128, 32, [1], [40001]),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("impl", [0, 1])
def test_matches_the_definition(shape, impl):
    check(*shape, impl, seed=len(shape[5]) + shape[4], extra_rows=3)


@pytest.mark.parametrize("shape", [(2, 4, 2, 32, 16, [5, 0, 70], [5, 9, 300]), (1, 4, 1, 128, 8, [9, 1], [100, 77]), (1, 3, 3, 64, 24, [4], [50]), (1, 8, 8, 32, 8, [1], [1])])
def test_shapes_of_the_plain_kernel(shape):
    check(*shape, None, seed=7, extra_rows=1)


def test_random_ragged_batches():
    rng = np.random.default_rng(42)
    for i in range(24):
        nkv, G = int(rng.choice([1, 2, 3])), int(rng.integers(1, 9))
        B = int(rng.integers(1, 12))
        kv = rng.integers(0, 1 + int(rng.choice([20, 300, 3000])), B)
        ql = np.minimum(rng.integers(0, 1 + int(rng.choice([2, 20, 300])), B), kv)
        kv[0], ql[0] = max(kv[0], 1), max(ql[0], 1)
        check(int(rng.integers(1, 4)), nkv * G, nkv, int(rng.choice([64, 128])), int(rng.choice([16, 32, 48, 64])), ql.tolist(), kv.tolist(), 0, seed=i)


@pytest.mark.parametrize("impl", [0, 1])
def test_hundreds_of_sequences(impl):
    """More sequences than a warp scans at once, most of them one token or none: a decode step in chunk form."""
    rng = np.random.default_rng(3)
    kv = rng.integers(0, 200, 515)
    ql = np.minimum(rng.choice([0, 1, 1, 1, 2, 130], 515), kv)
    kv[500:], ql[500:] = 0, 0                                 # the call's end owns nothing
    check(1, 4, 1, 64, 16, ql.tolist(), kv.tolist(), impl, seed=4)


def test_two_calls_at_once_with_a_scratch_each():
    import torch
    from paper_2602_07306_b200 import pt
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    calls = []
    for i, (ql, kl) in enumerate((([300, 1, 5], [3000, 900, 4000]), ([4, 4, 250], [5000, 40, 260]))):
        q, pool, bt = case(2, 8, 2, 128, 16, ql, kl, seed=20 + i)
        calls.append((d(q.reshape(2, sum(ql), -1)).bfloat16(), d(pool).bfloat16(), d(bt), d(np.array(ql, np.int32)), d(np.array(kl, np.int32))))
    kw = dict(nq=8, nkv=2, dh=128, ps=16)
    want = [pt.kernel_chunk_attn(*c, **kw)[0].clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    scratch = [pt.chunk_attn_scratch(2, 3, 8, 128, "cuda") for _ in calls]
    status = torch.zeros((2, 16), dtype=torch.int32, device="cuda")
    outs = [[torch.zeros_like(c[0]) for _ in range(10)] for c in calls]
    torch.cuda.synchronize()
    for r in range(10):
        for i, c in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                pt.kernel_chunk_attn(*c, **kw, out=outs[i][r], scratch=scratch[i], status=status[i])
    torch.cuda.synchronize()
    assert status.any().item() is False
    assert all(torch.equal(o, want[i]) for i in range(2) for o in outs[i])


@pytest.mark.parametrize("impl", [0, 1])
def test_scores_that_climb_and_large_scores(impl):
    """Running maxima that have to be raised again and again, and scores far beyond what exp2 takes unshifted."""
    T, nq, nkv, dh, ps, q_len, kv_len = 1, 4, 2, 128, 16, [6, 140], [900, 1700]
    q, pool, bt = case(T, nq, nkv, dh, ps, q_len, kv_len, seed=3, scale=0.5)
    for b, n in enumerate(kv_len):                             # every key points the queries' way, longer from tile to tile
        pos = np.arange(n)
        rise = (pos / n * 60)[:, None]
        u = np.zeros(dh, np.float32); u[0] = 1
        for h in range(nkv):
            pool[0, bt[b, pos // ps], 0, h, pos % ps] = I.round_to_bf16((pool[0, bt[b, pos // ps], 0, h, pos % ps] + rise * u).astype(np.float32))
    q[..., 0] = 4.0
    ref, bound = reference(q, pool, bt, q_len, kv_len, ps)
    got, status = call(q, pool, bt, q_len, kv_len, ps, impl)
    assert status == [0, 0] and np.all(np.abs(got - ref) <= bound)


@pytest.mark.parametrize("impl", [0, 1])
def test_bad_lengths_and_pages_are_reported(impl):
    q, pool, bt = case(1, 4, 2, 64, 16, [3, 5], [40, 60], seed=1)
    maxp = bt.shape[1]
    for ql, kl in (([3, -1], [40, 60]), ([3, 5], [2, 60]), ([3, 5], [40, maxp * 16 + 1]), ([3, 6], [40, 60]), ([2 ** 30, 2 ** 30], [2 ** 30, 2 ** 30]), ([3, 5], [40, -1])):
        got, status = call(q, pool, bt, ql, kl, 16, impl)
        assert status[0] == 8 and np.all(got == 5.0), (ql, kl)
    for bad in (-1, pool.shape[1], 2 ** 31 - 1, -2 ** 31):
        b2 = bt.copy()
        b2[1, 1] = bad
        got, status = call(q, pool, b2, [3, 5], [40, 60], 16, impl)
        assert status[0] == 8, bad
        good, _ = call(q, pool, bt, [3, 5], [40, 60], 16, impl)
        assert np.array_equal(got[:, :3], good[:, :3])          # the other sequence is not touched by it


def test_other_pages_for_the_same_tokens_and_repeats_give_the_same_bits():
    ql, kl = [9, 1, 150], [777, 3000, 1500]
    q, pool, bt = case(2, 8, 2, 128, 16, ql, kl, seed=5)
    got, _ = call(q, pool, bt, ql, kl, 16)
    again, _ = call(q, pool, bt, ql, kl, 16)
    perm = np.random.default_rng(0).permutation(pool.shape[1])
    pool2 = np.empty_like(pool)
    pool2[:, perm] = pool
    other, _ = call(q, pool2, np.where(bt >= 0, perm[np.maximum(bt, 0)], bt).astype(np.int32), ql, kl, 16)
    assert np.array_equal(got, again) and np.array_equal(got, other)


def test_a_captured_call_replays_with_other_lengths():
    import torch
    from paper_2602_07306_b200 import pt
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    ql, kl = [4, 4, 4], [700, 900, 300]
    q, pool, bt = case(1, 8, 2, 128, 16, ql, kl, seed=6)
    dq, dp, db = d(q.reshape(1, 12, -1)).bfloat16(), d(pool).bfloat16(), d(bt)
    dql, dkl = d(np.array(ql, np.int32)), d(np.array(kl, np.int32))
    out, scratch, status = torch.zeros_like(dq), pt.chunk_attn_scratch(1, 3, 8, 128, "cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    go = lambda: pt.kernel_chunk_attn(dq, dp, db, dql, dkl, nq=8, nkv=2, dh=128, ps=16, out=out, scratch=scratch, status=status)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        go()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            go()
    st.synchronize()
    for ql2, kl2 in ((ql, kl), ([1, 11, 0], [650, 899, 300]), ([0, 0, 12], [0, 1, 12])):
        dql.copy_(d(np.array(ql2, np.int32))); dkl.copy_(d(np.array(kl2, np.int32)))
        g.replay()
        torch.cuda.synchronize()
        ref, bound = reference(q, pool, bt, ql2, kl2, 16)
        got = out.float().cpu().numpy().astype(np.float64).reshape(1, 12, 8, 128)
        assert status[:2].tolist() == [0, 0] and np.all(np.abs(got - ref) <= bound)


def test_pool_views_with_a_larger_track_stride():
    """One layer of a [T, L, ...] pool: tracks are a layer count apart."""
    import torch
    from paper_2602_07306_b200 import pt
    ql, kl = [5, 2], [333, 90]
    q, pool, bt = case(3, 4, 2, 64, 16, ql, kl, seed=8)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    full = torch.full((3, 4) + pool.shape[1:], float("nan"), dtype=torch.bfloat16, device="cuda")
    full[:, 2] = d(pool).bfloat16()
    got, status = pt.kernel_chunk_attn(d(q.reshape(3, 7, -1)).bfloat16(), full[:, 2], d(bt), d(np.array(ql, np.int32)), d(np.array(kl, np.int32)), nq=4, nkv=2, dh=64, ps=16)
    want, _ = call(q, pool, bt, ql, kl, 16)
    assert status[:2].tolist() == [0, 0] and np.array_equal(got.float().cpu().numpy().astype(np.float64).reshape(want.shape), want)
