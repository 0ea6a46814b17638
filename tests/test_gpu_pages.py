"""Page copies, forked sequences with copy on write, compaction and moves of the pool on the GPU.  Copies are compared bit for
bit; forwards over shared, compacted or moved pages must give the same bits as over pages of their own (the kernels read the
same values in the same order)."""
import numpy as np
import pytest

from oracle import pt_oracle as O
from paper_2602_07306_b200 import inputs as I
from tests import helpers as Hp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,L,pages,width,dtype,n", [
    (1, 1, 2, 8, "bf16", 1),                   # one 16-byte page
    (1, 2, 5, 256, "bf16", 2),
    (2, 3, 9, 1000, "f32", 4),                 # pages that are no multiple of a warp's piece
    (3, 2, 40, 5 * 1024 + 8, "bf16", 17),
    (2, 2, 1300, 64, "bf16", 600),             # more pairs than one launch carries
    (1, 4, 7, 16, "u8", 3),
])
def test_copies_are_exact_and_touch_nothing_else(T, L, pages, width, dtype, n):
    import torch
    from paper_2602_07306_b200 import pt
    dt = {"bf16": torch.int16, "f32": torch.int32, "u8": torch.uint8}[dtype]
    g = torch.Generator(device="cuda").manual_seed(pages)
    pool = torch.randint(0, 127, (T, L, pages, width), dtype=dt, device="cuda", generator=g)
    r = np.random.default_rng(n).permutation(pages)
    src, dst = r[:n].copy(), r[n:2 * n].copy()
    if n > 2:
        src[1] = src[0]                        # one page read twice
    want = pool.clone()
    want[:, :, torch.from_numpy(dst).cuda()] = pool[:, :, torch.from_numpy(src).cuda()]
    other = torch.randint(0, 127, (T, L, pages + 3, width), dtype=dt, device="cuda", generator=g)
    want_o = other.clone()
    want_o[:, :, torch.from_numpy(dst).cuda()] = pool[:, :, torch.from_numpy(src).cuda()]
    pt.kernel_kv_copy_pages(pool, src, dst, out=other)
    pt.kernel_kv_copy_pages(pool, src, dst)
    pt.kernel_kv_copy_pages(pool, [], [])
    assert torch.equal(pool, want) and torch.equal(other, want_o)
    with pytest.raises(ValueError):
        pt.kernel_kv_copy_pages(pool, [0], [0, 1])
    with pytest.raises(ValueError):
        pt.kernel_kv_copy_pages(pool, [0], [1], out=other[:, :, :, : width // 2])
    with pytest.raises(pt.PtError):
        pt.kernel_kv_copy_pages(pool, [0, 0], [1, 1])


def test_offsets_beyond_32_bits():
    import torch
    from paper_2602_07306_b200 import pt
    pages, width = 70000, 64 * 1024            # 4.6e9 bytes in one slab
    pool = torch.zeros((1, 1, pages, width), dtype=torch.uint8, device="cuda")
    pool[0, 0, pages - 1] = 7
    pool[0, 0, 3] = 9
    pt.kernel_kv_copy_pages(pool, [pages - 1, 3], [5, pages - 2])
    assert torch.all(pool[0, 0, 5] == 7) and torch.all(pool[0, 0, pages - 2] == 9) and int(pool[0, 0, 6].sum()) == 0


def test_a_captured_copy_keeps_its_list():
    import torch
    from paper_2602_07306_b200 import pt
    pool = torch.arange(6 * 8, dtype=torch.int32, device="cuda").view(1, 1, 6, 8).clone()
    st = torch.cuda.Stream()
    src, dst = np.array([0, 1], np.int32), np.array([4, 5], np.int32)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            pt.kernel_kv_copy_pages(pool, src, dst)
    src[:], dst[:] = 3, 2
    pool[0, 0, 0] += 100
    st.wait_stream(torch.cuda.current_stream())
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(pool[0, 0, 4], pool[0, 0, 0]) and torch.equal(pool[0, 0, 5], pool[0, 0, 1])


CASES = {
    "bf16": dict(dtype="bf16", H=256, nq=4, nkv=2, kv="model", ps=16),
    "bf16_ps8": dict(dtype="bf16", H=128, nq=4, nkv=2, kv="model", ps=8),
    "f32": dict(dtype="f32", H=128, nq=4, nkv=4, kv="model", ps=8),
    "e4m3": dict(dtype="bf16", H=256, nq=2, nkv=1, kv="e4m3", ps=16),
}


def _model(c, seed=0):
    wl = I.Workload("pages", T=2, L=4, D=2, hidden=c["H"], heads=c["nq"], kv_heads=c["nkv"], ffn=352, dtype=c["dtype"], mode="prefill", batch=1, seq=8)
    ws = I.WeightSource(wl, std=0.05, gain_jitter=0.1)
    return wl, ws, Hp.make_model(wl, ws, max_pos=256)


def _x(wl, rng, *lead):
    x = rng.standard_normal((wl.T,) + lead + (wl.hidden,), dtype=np.float32)
    return I.round_to_bf16(x) if wl.dtype == "bf16" else x


@pytest.mark.parametrize("case", list(CASES))
def test_forked_sequences_continue_as_if_they_had_their_own_pages(case):
    import torch
    c = CASES[case]
    wl, ws, m = _model(c)
    rng = np.random.default_rng(1)
    ps, P, n_fork = c["ps"], 3 * c["ps"] + 5, 4
    x = Hp.to_dev(m, _x(wl, rng, 1, P))
    steps = [Hp.to_dev(m, _x(wl, rng, n_fork + 1)) for _ in range(ps + 3)]
    chunk = Hp.to_dev(m, _x(wl, rng, n_fork + 1, 7))
    # every sequence prefilled on its own
    own = m.new_cache(64, ps, kv_dtype=c["kv"])
    seqs = list(range(n_fork + 1))
    for s in seqs:
        m.prefill(own, x, [s])
    # one prefill, the others forked from it
    fk = m.new_cache(64, ps, kv_dtype=c["kv"])
    m.prefill(fk, x, [0])
    free0 = fk.free_pages()
    for s in seqs[1:]:
        fk.fork(0, s)
    assert fk.free_pages() == free0 and fk.block_table(3) == fk.block_table(0) and fk.page_refs(fk.block_table(0)[0]) == n_fork + 1
    for i, st in enumerate(steps):
        a, b = m.decode_step(own, st, seqs), m.decode_step(fk, st, seqs)
        assert torch.equal(a, b), i
        if i == 0:      # the shared last page: copied for all but one owner
            assert fk.free_pages() == free0 - n_fork and fk.page_refs(fk.block_table(0)[0]) == n_fork + 1
            assert len({fk.block_table(s)[3] for s in seqs}) == n_fork + 1
    assert torch.equal(m.prefill(own, chunk, seqs), m.prefill(fk, chunk, seqs))
    # a fork of a prefix that ends inside a page, then truncation into shared pages
    fk.fork(2, 9, ps + 3); own.fork(2, 9, ps + 3)
    fk.truncate(2, 2 * ps + 1); own.truncate(2, 2 * ps + 1)
    one = Hp.to_dev(m, _x(wl, rng, 2, 5))
    assert torch.equal(m.prefill(own, one, [9, 2]), m.prefill(fk, one, [9, 2]))
    st = Hp.to_dev(m, _x(wl, rng, n_fork + 2))
    assert torch.equal(m.decode_step(own, st, seqs + [9]), m.decode_step(fk, st, seqs + [9]))
    for s in seqs + [9]:
        fk.release(s)
    assert fk.free_pages() == 64 and all(fk.page_refs(p) == 0 for p in range(64))
    assert m.device_status() == (0, 0)
    m.close()


def test_forked_sequences_follow_the_oracle():
    wl, ws, m = _model(CASES["f32"])
    cfg = Hp.oracle_cfg(wl)
    rng = np.random.default_rng(2)
    x, y, z = _x(wl, rng, 1, 21), _x(wl, rng, 2, 6), _x(wl, rng, 2)
    c, oc = m.new_cache(20, 8), O.PagedKVCache(cfg, 20, 8)
    m.prefill(c, Hp.to_dev(m, x), [0]); O.pt_prefill(cfg, ws, x, oc, [0])
    c.fork(0, 1, 13); oc.fork(0, 1, 13)
    Hp.assert_close(m.prefill(c, Hp.to_dev(m, y), [0, 1]).cpu().numpy(), O.pt_prefill(cfg, ws, y, oc, [0, 1]), "f32")
    Hp.assert_close(m.decode_step(c, Hp.to_dev(m, z), [1, 0]).cpu().numpy(), O.pt_decode_step(cfg, ws, z, oc, [1, 0]), "f32")
    m.close()


def test_a_full_cache_refuses_the_copy_and_stays_as_it_was():
    import torch
    from paper_2602_07306_b200 import pt
    wl, ws, m = _model(CASES["bf16"])
    rng = np.random.default_rng(3)
    c = m.new_cache(3, 16)
    m.prefill(c, Hp.to_dev(m, _x(wl, rng, 1, 40)), [0])       # three pages: none left
    c.fork(0, 1)
    st = Hp.to_dev(m, _x(wl, rng, 1))
    with pytest.raises(pt.PtError) as e:
        m.decode_step(c, st, [1])
    assert e.value.code == 5 and c.length(1) == 40 and c.block_table(1) == c.block_table(0) and c.page_refs(2) == 2
    with pytest.raises(pt.PtError):
        m.decode_step(c, Hp.to_dev(m, _x(wl, rng, 2)), [0, 1])
    c.release(0)                                              # now the sequence is alone on its pages
    m.decode_step(c, st, [1])
    assert c.length(1) == 41 and m.device_status() == (0, 0)
    m.close()


@pytest.mark.parametrize("case", list(CASES))
def test_compaction_and_moves_keep_every_sequence(case):
    import torch
    c = CASES[case]
    wl, ws, m = _model(c, seed=1)
    rng = np.random.default_rng(4)
    ps, pages = c["ps"], 40
    order = I.free_list_permutation(pages, seed=6)
    a, b = m.new_cache(pages, ps, order, kv_dtype=c["kv"]), m.new_cache(pages, ps, order, kv_dtype=c["kv"])
    x = Hp.to_dev(m, _x(wl, rng, 5, 4 * ps + 3))
    for k in (a, b):
        m.prefill(k, x, [0, 1, 2, 3, 4])
        k.fork(1, 7, 2 * ps)
        for s in (0, 1, 3):
            k.release(s)
    used = pages - a.free_pages()
    tables = {s: a.block_table(s) for s in (2, 4, 7)}
    moved = a.compact()
    assert moved == len({p for t in tables.values() for p in t if p >= used})
    assert sorted({p for s in tables for p in a.block_table(s)}) == list(range(used)) and a.free_pages() == pages - used
    for s, t in tables.items():                               # pages below the border stay where they were
        assert [q for p, q in zip(t, a.block_table(s)) if p < used] == [p for p in t if p < used]
    assert a.compact() == 0
    st = Hp.to_dev(m, _x(wl, rng, 3))
    assert torch.equal(m.decode_step(a, st, [2, 4, 7]), m.decode_step(b, st, [2, 4, 7]))
    used = pages - a.free_pages()
    for size in (used, 64):                                   # to the smallest pool, then to a larger one
        a.resize(size)
        assert a.num_pages == size and a.free_pages() == size - used
    st = Hp.to_dev(m, _x(wl, rng, 3, 9))
    assert torch.equal(m.prefill(a, st, [7, 2, 4]), m.prefill(b, st, [7, 2, 4]))
    from paper_2602_07306_b200 import pt
    with pytest.raises(pt.PtError) as e:
        a.resize(3)
    assert e.value.code == 5 and a.num_pages == 64
    st = Hp.to_dev(m, _x(wl, rng, 2))
    assert torch.equal(m.decode_step(a, st, [7, 4]), m.decode_step(b, st, [7, 4]))
    assert m.device_status() == (0, 0)
    m.close()
