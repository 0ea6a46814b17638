"""Forward calls on a cache in the 4-bit format against the oracle with the same format.

The device quantises the K and V that its bf16 GEMM produced, the oracle its exact ones: a value near a code boundary lands on
the neighbouring code.  That and the rounding of the contractions' operands is measured on the very rows of the run, inside the
oracle's own arithmetic (as tests/bf16_floor.py does for the other formats), and what the device is allowed is that floor times
its margin for the mean; for the largest error, which is one draw of a tail on either side, three times the floor's largest."""
import numpy as np
import pytest

from oracle import kv4
from oracle import pt_oracle as O
from paper_2602_07306_b200 import inputs as I
from tests import bf16_floor as F
from tests import helpers as Hp

pytestmark = pytest.mark.gpu


@pytest.fixture
def four(monkeypatch):
    """The oracle's coded cache holds this format's values, its scales are ones."""
    def q(v):
        x = kv4.values(*kv4.quantize(v))
        return x, np.ones(x.shape[:-1] + (1,))
    monkeypatch.setattr(O, "kv_quantize", q)


def setup(H, nq, nkv, T=2, L=4, D=2, max_pos=900):
    wl = I.Workload("kv4", T=T, L=L, D=D, hidden=H, heads=nq, kv_heads=nkv, ffn=352, dtype="bf16", mode="prefill", batch=1, seq=8)
    ws = I.WeightSource(wl, gain_jitter=0.1)
    return wl, ws, Hp.make_model(wl, ws, max_pos=max_pos)


def draw(wl, rng, *lead):
    return I.round_to_bf16(rng.standard_normal((wl.T,) + lead + (wl.hidden,), dtype=np.float32))


def floor(wl, ws, history):
    """(max, mean) relative error over all rows that rounding alone leaves."""
    worst = err = size = top = 0.0
    for x in history:
        h = {}
        for rnd in (False, True):
            cur = [x[t] for t in range(wl.T)]
            for l in range(wl.L):
                cur = [F._layer(cur[t], ws.get(t, l), np.arange(x.shape[1]), wl.heads, wl.kv_heads, wl.head_dim, rnd, True) for t in range(wl.T)]
                if (l + 1) % wl.D == 0:
                    cur = [sum(cur)] * wl.T
            h[rnd] = cur[0]
        d = np.abs(h[True] - h[False])
        worst, err, size, top = max(worst, d.max()), err + d.sum(), size + np.abs(h[False]).sum(), max(top, np.abs(h[False]).max())
    return worst / top, err / size


class Run:
    """The library's calls beside the oracle's, and the errors of all rows at the end."""

    def __init__(self, wl, ws, m, ps, pages):
        order = I.free_list_permutation(pages, seed=2)
        self.wl, self.ws, self.m, self.cfg = wl, ws, m, Hp.oracle_cfg(wl)
        self.c, self.oc = m.new_cache(pages, ps, order, kv_dtype="e2m1"), O.PagedKVCache(self.cfg, pages, ps, order, kv_format="e4m3")
        self.c.pool.zero_()
        self.history, self.got, self.ref = {}, [], []

    def _note(self, x, n, ids, got, ref):
        assert np.isfinite(got).all()
        self.got.append(got.reshape(-1, self.wl.hidden)); self.ref.append(ref.reshape(-1, self.wl.hidden))
        for e, k, s in zip(np.cumsum(n), n, ids):
            self.history[s] = np.concatenate([self.history.get(s, np.zeros((self.wl.T, 0, self.wl.hidden))), x[:, e - k:e].astype(np.float64)], 1)
            assert self.c.length(s) == self.oc.length[s] and self.c.block_table(s) == self.oc.block_table[s]

    def prefill(self, x, ids):
        B, S = x.shape[1:3]
        got = self.m.prefill(self.c, Hp.to_dev(self.m, x), ids).cpu().numpy()
        self._note(x.reshape(self.wl.T, B * S, -1), [S] * B, ids, got, O.pt_prefill(self.cfg, self.ws, x, self.oc, ids))

    def decode(self, x, ids):
        got = self.m.decode_step(self.c, Hp.to_dev(self.m, x), ids).cpu().numpy()
        self._note(x, [1] * len(ids), ids, got, O.pt_decode_step(self.cfg, self.ws, x, self.oc, ids))

    def extend(self, x, n, ids):
        got = self.m.extend(self.c, Hp.to_dev(self.m, x), n, ids).cpu().numpy()
        self._note(x, n, ids, got, O.pt_extend(self.cfg, self.ws, x.astype(np.float64), n, self.oc, ids))

    def check(self, name):
        assert self.m.device_status() == (0, 0)
        fmx, fmean = floor(self.wl, self.ws, self.history.values())
        mx, mean = Hp.rel_errs(np.concatenate(self.got), np.concatenate(self.ref))
        Hp.record(f"e2m1 cache, {name}", mx, mean, max(2e-2, 3 * fmx), max(2e-3, F.FLOOR_MARGIN * fmean))
        assert mean <= max(2e-3, F.FLOOR_MARGIN * fmean) and mx <= max(2e-2, 3 * fmx), (mx, fmx, mean, fmean)

    def check_pool(self):
        """Cached values: nearly all the oracle's, the others a code or a scale away; nothing outside the sequences."""
        deq = self.c.dequantized().cpu().numpy().astype(np.float64)
        mine = np.zeros(deq.shape[2], bool)
        same = []
        for s in self.history:
            pos = np.arange(self.c.length(s))
            pg, sl = np.array(self.c.block_table(s))[pos // self.c.page_size], pos % self.c.page_size
            opg, osl = self.oc._pages_slots(s, pos)
            a, b = deq[:, :, pg, :, :, sl], self.oc.pool[:, :, opg, :, :, osl]
            same.append((a == b).mean())
            top = np.abs(b).reshape(b.shape[:-1] + (-1, 32)).max(-1).repeat(32, -1)
            assert (np.abs(a - b) <= 0.75 * top + 1e-30).all()
            mine[pg] = True
        assert np.mean(same) > 0.9, same
        assert not deq[:, :, ~mine].any()


@pytest.mark.parametrize("H,nq,nkv,ps", [(256, 2, 2, 16), (512, 4, 1, 32), (128, 2, 1, 48), (256, 4, 4, 16), (1024, 8, 1, 16)])
def test_prefill_decode_and_ragged_calls_follow_the_oracle(four, H, nq, nkv, ps):
    wl, ws, m = setup(H, nq, nkv)
    rng = np.random.default_rng(3)
    r = Run(wl, ws, m, ps, 2000 // ps + 20)
    r.prefill(draw(wl, rng, 3, 150), [0, 3, 7])                 # a prompt: the bf16 copy
    r.prefill(draw(wl, rng, 3, 7), [7, 0, 3])                   # a few tokens on a context: from the codes
    for _ in range(2):
        r.decode(draw(wl, rng, 3), [0, 7, 3])
    n, ids = [1, 4, 130, 1], [0, 3, 9, 7]                       # tokens beside a prompt's chunk
    r.extend(draw(wl, rng, sum(n)), n, ids)
    n, ids = [5, 1, 3], [7, 9, 0]                               # speculated tokens
    r.extend(draw(wl, rng, sum(n)), n, ids)
    r.decode(draw(wl, rng, 4), [9, 0, 3, 7])
    r.check(f"hidden {H}, heads {nq}/{nkv}, pages of {ps}")
    r.check_pool()
    m.close()


def test_forks_copies_on_write_compaction_and_moves(four):
    wl, ws, m = setup(256, 2, 1)
    rng = np.random.default_rng(5)
    r = Run(wl, ws, m, 16, 60)
    r.prefill(draw(wl, rng, 1, 45), [0])
    for dst in (1, 2):
        r.c.fork(0, dst)
        r.oc.fork(0, dst, 45)
        r.history[dst] = r.history[0]
    x = draw(wl, rng, 3)

    def decode():
        got = m.decode_step(r.c, Hp.to_dev(m, draw_ := draw(wl, rng, 3)), [0, 1, 2]).cpu().numpy()
        ref = O.pt_decode_step(r.cfg, r.ws, draw_, r.oc, [0, 1, 2])
        for i in range(3):
            r.history[i] = np.concatenate([r.history[i], draw_[:, i:i + 1].astype(np.float64)], 1)
        r.got.append(got); r.ref.append(ref)
    decode()
    r.c.release(1); r.oc.release(1)
    del r.history[1]
    assert r.c.compact() >= 0
    r.c.resize(40)
    r.c.fork(0, 1)
    r.oc.fork(0, 1, 46)
    r.history[1] = r.history[0]
    decode()
    decode()
    r.check("forks, compaction, move")
    m.close()


def test_a_cache_of_each_format_shares_one_workspace():
    """Calls on caches of the three formats in turn, with the workspace of the largest."""
    wl, ws, m = setup(256, 2, 1)
    rng = np.random.default_rng(6)
    x, d = Hp.to_dev(m, draw(wl, rng, 2, 40)), Hp.to_dev(m, draw(wl, rng, 2))
    alone = {}
    for turn in range(2):
        for kv in ("model", "e4m3", "e2m1"):
            c = m.new_cache(20, 16, kv_dtype=kv)
            out = [m.prefill(c, x, [0, 1]).cpu().numpy(), m.decode_step(c, d, [0, 1]).cpu().numpy(), m.extend(c, d, [1, 1], [1, 0]).cpu().numpy()]
            if turn:
                assert all(np.array_equal(a, b) for a, b in zip(out, alone[kv]))
            alone[kv] = out
    assert m.device_status() == (0, 0)
    m.close()
