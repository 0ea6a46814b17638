"""Attention from the 4-bit codes where the softmax weights and the scales of V spread far: what fp16 products may lose.

A weight w (2^8 to 2^14 for the largest of a part of the keys) and a scale s of V meet in one fp16 product, the scale divided by the
power of two 2^E that its group of 32 columns has in its tile of 32 keys: the tile's largest scale of the group is then in [2^-5, 2).
Beside the roundings that tests/test_gpu_kv4.py counts, a key may so lose, relative to the row's largest softmax weight p_max and
to the largest scale S of its own tile and group (codes reach 6, 2^E <= 2^5 S):
  2^-25 of the weight below fp16's normal range, times s / 2^E < 2, and 2^-25 of the product:  3 * 2^-25 * 6 * 2^5 S * p_max / 2^8
  2^-25 of a scale that far below the tile's largest:                                          2^-25 * 6 * 2^5 S * p
but no more than seven times its own share p |v|: each of the three roundings to nearest errs by its number at most.
No group is held to another's scales, and none to those of other tiles."""
import numpy as np
import pytest

from paper_2602_07306_b200 import inputs as I
from tests.test_gpu_kv4 import attend, cache, queries

pytestmark = pytest.mark.gpu
TILE = 32


def reference(q, values, bt, q_len, kv_len, ps):
    """(out, bound) float64 [T, rows, nq, dh]."""
    import torch
    T, _, nq, dh = q.shape
    nkv = values.shape[3]
    G = nq // nkv
    out = torch.zeros((T, sum(q_len), nq, dh), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    dq, dv = torch.from_numpy(q).cuda().double(), torch.from_numpy(values).cuda()
    r = 0
    for b, (S, K) in enumerate(zip(q_len, kv_len)):
        pos = torch.arange(K, device="cuda")
        pg = torch.from_numpy(bt[b].astype(np.int64)).cuda()[pos // ps]
        seen = pos[None] <= torch.arange(K - S, K, device="cuda")[:, None]
        for h in range(nkv if S else 0):
            k, v = (dv[:, pg, i, h, pos % ps][:, None] for i in (0, 1))                          # [T, 1, K, dh]
            a = dq[:, r:r + S, h * G:(h + 1) * G].transpose(1, 2)                                # [T, G, S, dh]
            s = a @ k.transpose(-1, -2) / np.sqrt(dh)
            e = a.abs() @ k.abs().transpose(-1, -2) / np.sqrt(dh)
            tiny = 2.0 ** -38 * a.abs().amax(-1, keepdim=True) * k.abs().sum(-1)[:, :, None] / np.sqrt(dh)
            err = (2 * dh * 2.0 ** -24 * e + tiny + 2.0 ** -23 * s.abs() + 2.0 ** -21).masked_fill(~seen, 0).amax(-1, keepdim=True)
            p = torch.softmax(s.masked_fill(~seen, -np.inf), -1)
            o, A = p @ v, p @ v.abs()
            # an upper bound of each group's scale (its largest code is 3 at least, or the scale is the smallest), largest in each tile
            pad = torch.nn.functional.pad(v.abs(), (0, 0, 0, -K % TILE)).reshape(T, 1, -1, TILE, dh // 32, 32)
            top = (pad.amax((3, 5)) / 3 + 2.0 ** -17).repeat_interleave(TILE, 2)[:, :, :K].repeat_interleave(32, -1)
            floor = torch.zeros_like(o)
            for g in range(G):
                for i in range(S):
                    pk = p[:, g, i, :, None]
                    lost = torch.minimum((pk.amax(1, keepdim=True) * (3 * 6 * 2.0 ** (5 - 25 - 8)) + pk * (6 * 2.0 ** (5 - 25))) * top[:, 0], 7 * pk * v[:, 0].abs())
                    floor[:, g, i] = lost.masked_fill(~seen[i, :, None], 0).sum(1)
            lim = 2.0 ** -8 * o.abs() + (A * (2.0 ** -10 + 2.5 * err + 2 * K * 2.0 ** -24) + floor) * (1 + 2.0 ** -7)
            out[:, r:r + S, h * G:(h + 1) * G] = o.transpose(1, 2)
            bound[:, r:r + S, h * G:(h + 1) * G] = lim.transpose(1, 2)
        r += S
    return out.cpu().numpy(), bound.cpu().numpy()


def check(nq, nkv, dh, q_len, kv_len, q, make, seed=3, ps=64):
    """One sequence, alone (its keys are cut into many parts) and as many that share its pages (a warp has all keys of one)."""
    ql = [1] * len(kv_len) if q_len is None else q_len
    pool, values, bt = cache(1, nkv, dh, ps, kv_len, seed, make=make)
    want, bound = reference(q, values, bt, ql, kv_len, ps)
    for copies in (1, 1776):
        got, st = attend(np.tile(q, (1, copies, 1, 1)), pool, np.tile(bt, (copies, 1)), kv_len * copies, q_len and q_len * copies, ps, nkv)
        got = got.view((copies,) + want.shape[1:]) if copies > 1 else got
        d = np.abs(got.float().cpu().numpy().astype(np.float64) - want).max(0, keepdims=True)
        assert st == [0, 0] and np.isfinite(d).all()
        assert (d <= bound).all(), (copies, float((d / np.maximum(bound, 1e-300)).max()), float(np.abs(d / np.maximum(np.abs(want), 1e-300)).max()))
    return want, bound


def sink(K, dh, ps, v_of, at=5):
    """Keys of which the one at `at` has 2^gap times the weight of the others for the queries of peaked(gap); v_of(v) makes the values."""
    pos = np.arange(K)

    def make(x, bt):
        pg, sl = bt[0, pos // ps], pos % ps
        x[0, 0, pg, 0, sl] *= 0.02
        x[0, 0, pg[at], 0, sl[at], :32] = 1.0
        v = x[1, 0, pg, 0, sl]
        v_of(v)
        x[1, 0, pg, 0, sl] = v
    return make


def peaked(rows, nq, dh, gap, seed=3):
    q = queries(1, rows, nq, dh, seed, 0.05)
    q[..., :32] = np.float32(gap * np.log(2) * np.sqrt(dh) / 32)
    return I.round_to_bf16(q)


SHAPES = [(8, 1, 128, None), (8, 1, 128, [2]), (8, 1, 128, [3]), (1, 1, 64, None), (4, 1, 64, [4]), (4, 1, 64, [6])]      # one, two and three row tiles


@pytest.mark.parametrize("gap", [14, 17])
@pytest.mark.parametrize("nq,nkv,dh,q_len", SHAPES)
def test_small_values_behind_a_dominant_key(nq, nkv, dh, q_len, gap):
    """Scales of V of 2^-17 to 2^-13 under thousands of small weights: their sum is a good part of the output."""
    K = 8000

    def v_of(v):
        v[:] = np.exp2(-15 + np.arange(K) % 3 * 2.0)[:, None] * (1 + 0.2 * v)
        v[5] *= 0.01
    want, bound = check(nq, nkv, dh, q_len, [K], peaked(sum(q_len or [1]), nq, dh, gap), sink(K, dh, 64, v_of))
    assert (bound < 0.2 * np.abs(want)).all()                       # and the bound says something


@pytest.mark.parametrize("at", [5, 7, 7999])
@pytest.mark.parametrize("nq,nkv,dh,q_len", SHAPES)
def test_a_large_group_of_one_token_leaves_the_others(nq, nkv, dh, q_len, at):
    """One token has a group of values of 2^17, its other groups and all other tokens are ordinary."""
    K = 8000

    def v_of(v):
        v[:] = 0.4 * (1 + 0.2 * v)
        v[5] *= 0.01
        v[at, 32:64] = 2.0 ** 17
    want, bound = check(nq, nkv, dh, q_len, [K], peaked(sum(q_len or [1]), nq, dh, 16), sink(K, dh, 64, v_of))
    rest = np.r_[:32, 64:dh]
    assert (bound[..., rest] < 0.05 * np.abs(want[..., rest])).all()


@pytest.mark.parametrize("nq,nkv,dh,q_len", SHAPES)
def test_a_large_token_that_hardly_counts_leaves_the_other_tiles(nq, nkv, dh, q_len):
    """The first token has values of 2^17 and next to no weight: the same columns of the others keep theirs."""
    K = 8000

    def v_of(v):
        v[:] = 0.02 * (1 + 0.2 * v)
        v[0] = 2.0 ** 17
        v[70] *= 0.01

    def make(x, bt):
        sink(K, dh, 64, v_of, at=70)(x, bt)
        x[0, 0, bt[0, 0], 0, 0, :32] = -2.0                          # 2^-34 of the others' weight
    want, bound = check(nq, nkv, dh, q_len, [K], peaked(sum(q_len or [1]), nq, dh, 17), make)
    assert (bound < 0.05 * np.abs(want)).all()


@pytest.mark.parametrize("nq,nkv,dh,q_len", SHAPES)
def test_scales_that_rise_and_fall_from_tile_to_tile(nq, nkv, dh, q_len):
    K = 3000
    def make(x, bt):
        pos = np.arange(K)
        pg, sl = bt[0, pos // 64], pos % 64
        x[1, 0, pg, 0, sl] *= np.exp2((pos // 32 * 7) % 23 - 11.0)[:, None]
        x[1, 0, pg, 0, sl, 32:64] *= np.exp2(-((pos // 32 * 5) % 9.0))[:, None]
        x[1, 0, pg, 0, sl, :32] *= (pos // 64 % 3 > 0)[:, None]      # and tiles of zeros
    check(nq, nkv, dh, q_len, [K], queries(1, sum(q_len or [1]), nq, dh, 3), make)


@pytest.mark.parametrize("T,nq,nkv,dh,ps,q_len,kv_len", [
    (2, 8, 2, 128, 16, [4], [301]), (1, 16, 2, 128, 32, [2, 2], [700, 5]), (2, 8, 1, 64, 64, [2, 1, 3], [5000, 40, 33]), (1, 5, 1, 128, 48, [3], [1500]),
    (3, 6, 2, 64, 16, [4, 5, 3, 0, 4], [47, 96, 333, 9, 64]), (1, 8, 1, 128, 16, [2] * 40, [20 + (977 * i) % 900 for i in range(40)]), (2, 9, 9, 128, 16, [16, 12], [16, 2000])])
def test_two_row_tiles(T, nq, nkv, dh, ps, q_len, kv_len):
    """Calls whose sequences have 9 to 16 (token, head) rows on average, element by element."""
    rows = sum(q_len) * (nq // nkv) / len(q_len)
    assert 8 < rows <= 16
    pool, values, bt = cache(T, nkv, dh, ps, kv_len, 7)
    q = queries(T, sum(q_len), nq, dh, 7)
    want, bound = reference(q, values, bt, q_len, kv_len, ps)
    got, st = attend(q, pool, bt, kv_len, q_len, ps, nkv)
    d = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    assert st == [0, 0] and np.isfinite(d).all() and (d <= bound).all(), float((d / np.maximum(bound, 1e-300)).max())
