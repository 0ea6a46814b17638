"""Workloads of the 4-bit KV cache (E2M1 codes, one 8-bit scale for 32 of them), with their plain forms.

Three operators that a server needs to keep the context of its users in a quarter of the bytes:

  write   new tokens' K and V quantised into the cache's pages (optionally with the values that the cache then holds)
  read    cached sequences back into pages of a bf16 cache, which every other attention of the library reads
  attn    attention of one or a few new tokens per sequence straight from the 4-bit pages

A cached vector (one token, one KV head, K or V) of dh values is split into groups of 32.  A group's scale s is the smallest
unsigned E5M3 number (the upper 8 bits of a positive fp16, at most 61440) with max|v| <= 6 s, and a code is v / s rounded to
the nearest E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign), ties to the even code, saturating.  A group with a NaN or an
infinity has the scale byte 255 (a NaN) and codes of zero.  A page is [kv_head][slot / 16] blocks of 16 tokens' K and V:

  K codes    slot s at place (s % 2) * 8 + s / 2 of dh / 2 bytes; within: [q < 4][group][8 codes of dims 32 group + 8 q ..]
  K scales   [slot][group]
  V codes    per slot s = 4 q + i and g < 8: [group][4 codes of dims 32 group + 4 g ..]; dh 128: [i / 2][g][q][i % 2], dh 64: [g][q][i]
  V scales   [q][group][i]

``run`` computes the plain form in elementary torch operations, or, with ``own`` set, makes the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"

# ---------------------------------------------------------------------------------------------- cases


def listed():
    return [
        # a decode step of eight users on the small model: latency
        dict(name="write_8_tokens_small", op="write", T=4, M=8, nkv=8, dh=64, ps=16, values=False, skip=0.0, run=1),
        # a decode step of the batched decode workload (8 tracks, 64 sequences): one token into a page of each
        dict(name="write_decode_64", op="write", T=8, M=64, nkv=8, dh=128, ps=16, values=False, skip=0.0, run=1),
        # a ragged step with rows that are not cached (padding), odd sizes, grouped heads
        dict(name="write_ragged_777", op="write", T=3, M=777, nkv=2, dh=128, ps=48, values=True, skip=0.1, run=37),
        # prompts of 8192 tokens in all, with the rounded values for the attention of the same call
        dict(name="write_prompt_8192", op="write", T=8, M=8192, nkv=8, dh=128, ps=16, values=True, skip=0.0, run=4096),
        # one short context of the small model read back: latency
        dict(name="read_1x301_small", op="read", T=4, B=1, nkv=8, dh=64, ps=16, ops=16, kv_lo=301, kv_hi=301, lens=1),
        # the contexts of a mixed batch into 16-token pages in front of a chunk of a prompt
        dict(name="read_mixed_28", op="read", T=4, B=28, nkv=4, dh=128, ps=32, ops=16, kv_lo=800, kv_hi=4096, lens=4),
        # four long contexts (a cache changes its format)
        dict(name="read_4x16k", op="read", T=8, B=4, nkv=4, dh=128, ps=64, ops=32, kv_lo=9000, kv_hi=16384, lens=5),
        # one user, a short context, the small model: latency
        dict(name="attn_1x301_small", op="attn", T=4, B=1, nq=8, nkv=8, dh=64, ps=16, q="one", q_hi=1, kv_lo=301, kv_hi=301, lens=1),
        # speculated tokens of eight users at the decode workload's shape, idle sequences among them
        dict(name="attn_verify_8x2k", op="attn", T=8, B=8, nq=8, nkv=8, dh=128, ps=16, q="ragged", q_hi=8, kv_lo=1800, kv_hi=2300, lens=2),
        # one user with a prompt of 63488 tokens on the paper's head layout (8 query heads on one KV head)
        dict(name="attn_1x63488", op="attn", T=8, B=1, nq=8, nkv=1, dh=128, ps=64, q="one", q_hi=1, kv_lo=63488, kv_hi=63488, lens=3),
        # few users with long contexts, grouped heads, five tokens each to check
        dict(name="attn_verify_4x30k", op="attn", T=4, B=4, nq=16, nkv=4, dh=128, ps=32, q="fixed", q_hi=5, kv_lo=9000, kv_hi=31000, lens=4),
        # the ragged decode workload: 256 sequences, one token each
        dict(name="attn_decode_256_ragged", op="attn", T=4, B=256, nq=16, nkv=4, dh=128, ps=16, q="one", q_hi=1, kv_lo=512, kv_hi=2048, lens=6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attn", "attn"])
    T, dh, ps = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128, 128]), rng.choice([16, 32, 48, 64])
    if op == "write":
        c = dict(op=op, T=T, M=_log(rng, 1, 8192), nkv=rng.choice([1, 2, 3, 4, 8]), dh=dh, ps=ps, values=rng.random() < 0.5,
                 skip=rng.choice([0.0, 0.0, 0.2]), run=1)
        c["run"] = _log(rng, 1, c["M"])
        return c
    c = dict(op=op, T=T, B=_log(rng, 1, 200), nkv=rng.choice([1, 2, 3, 4, 8]), dh=dh, ps=ps, kv_lo=0, kv_hi=_log(rng, 20, 60000), lens=rng.randrange(1 << 20))
    if op == "read":
        c["ops"] = rng.choice([8, 16, 24, 32, 64])
        most = 2.0e8
    else:
        c["nq"] = c["nkv"] * rng.choice([1, 2, 3, 4, 5, 8])
        c["q"] = rng.choice(["one", "one", "fixed", "ragged"])
        c["q_hi"] = 1 if c["q"] == "one" else _log(rng, 1, 8)
        most = 8.0e8
    c["kv_hi"] = max(c["kv_hi"], c.get("q_hi", 1) + 1)
    # no more than the largest listed case
    while c["B"] > 1 and c["T"] * c["B"] * c["nkv"] * c["kv_hi"] * 2 * dh > most:
        c["B"] = (c["B"] + 1) // 2
    while c["T"] * c["B"] * c["nkv"] * c["kv_hi"] * 2 * dh > most:
        c["kv_hi"] = max(20, c["kv_hi"] * 2 // 3)
    c["kv_lo"] = rng.randint(1, c["kv_hi"])
    return c


def _lens(c):
    """New tokens and cached keys of every sequence of a case: plain lists, from the case alone."""
    r = random.Random(c["lens"])
    kv = [r.randint(c["kv_lo"], c["kv_hi"]) for _ in range(c["B"])]
    kind = c.get("q", "one")
    q = [r.randint(0, c["q_hi"]) for _ in kv] if kind == "ragged" else [c["q_hi"] if kind == "fixed" else 1] * c["B"]
    q[0] = max(1, q[0])
    return [min(a, b) for a, b in zip(q, kv)], kv


def _block_bytes(dh):
    return 2 * (16 * dh // 2 + 16 * dh // 32)


# ---------------------------------------------------------------------------------------------- the format, plain


def _scales():
    """The scale that each byte stands for (255: NaN)."""
    return (torch.arange(256, dtype=torch.int32, device=DEV) << 7).to(torch.int16).view(torch.float16).float()


def _quantise(x):
    """x float32 [..., dh] -> codes uint8 [..., dh], scale bytes uint8 [..., dh / 32]."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = g.abs().amax(-1)
    bad = ~torch.isfinite(amax)                                                      # a NaN makes the maximum a NaN
    value = _scales()
    byte = torch.searchsorted(value[:248] * 6, torch.where(bad, 0.0, amax).contiguous()).clamp_(max=247)
    s = value[byte][..., None]
    a = g.abs()
    code = (a > s * 0.25).to(torch.uint8)
    for bound, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= s * bound) if closed else (a > s * bound)
    code = torch.where(s > 0, code, 0) + torch.signbit(g).to(torch.uint8) * 8
    code = torch.where(bad[..., None], 0, code).to(torch.uint8)
    return code.reshape(x.shape), torch.where(bad, 255, byte).to(torch.uint8)


def _values(code, byte):
    """What codes [..., dh] and scale bytes [..., dh / 32] stand for, float32."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    v = grid[code.int()].view(*byte.shape, 32) * _scales()[byte.int()][..., None]
    return v.view(code.shape)


def _pack(k, ks, v, vs):
    """Codes uint8 [N, 16, dh] and scale bytes [N, 16, dh / 32] of K and V -> blocks uint8 [N, bytes]."""
    n, _, dh = k.shape
    nib = lambda a: (a[..., 0] | a[..., 1] << 4).reshape(n, -1)                       # noqa: E731
    kb = nib(k.view(n, 8, 2, dh // 32, 4, 4, 2).permute(0, 2, 1, 4, 3, 5, 6))
    v = v.view(n, 4, 2, 2, dh // 32, 8, 2, 2)                                        # q, i / 2, i % 2, group, g, pair, code
    vb = nib(v.permute(0, 2, 5, 1, 3, 4, 6, 7) if dh == 128 else v.permute(0, 5, 1, 2, 3, 4, 6, 7))
    return torch.cat([kb, ks.reshape(n, -1), vb, vs.view(n, 4, 4, -1).transpose(2, 3).reshape(n, -1)], 1)


def _unpack(block, dh):
    """Blocks uint8 [..., bytes] -> K and V float32 [..., 16, dh]."""
    lead, n = block.shape[:-1], block.shape[:-1].numel()
    kb, ks, vb, vs = block.reshape(n, -1).split([8 * dh, dh // 2, 8 * dh, dh // 2], 1)
    two = lambda a: torch.stack([a & 15, a >> 4], -1)                                 # noqa: E731
    k = two(kb).view(n, 2, 8, 4, dh // 32, 4, 2).permute(0, 2, 1, 4, 3, 5, 6).reshape(n, 16, dh)
    v = two(vb)
    v = v.view(n, 2, 8, 4, 2, dh // 32, 2, 2).permute(0, 3, 1, 4, 5, 2, 6, 7) if dh == 128 else v.view(n, 8, 4, 2, 2, dh // 32, 2, 2).permute(0, 2, 3, 4, 5, 1, 6, 7)
    vs = vs.view(n, 4, -1, 4).transpose(2, 3).reshape(n, 16, -1)
    return (_values(a, b).view(*lead, 16, dh) for a, b in ((k, ks.view(n, 16, -1)), (v.reshape(n, 16, dh), vs)))


# ---------------------------------------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"write": _prepare_write, "read": _prepare_read, "attn": _prepare_attn}[case["op"]](case, seed, g)


def _channels(c, g):
    """Magnitudes of K's channels: a few are far larger than the others, as in trained models."""
    wide = torch.rand((c["nkv"], c["dh"]), device=DEV, generator=g) < 0.04
    return torch.where(wide, 6.0, 1.0)


def _prepare_write(c, seed, g):
    T, M, nkv, dh, ps = (c[a] for a in ("T", "M", "nkv", "dh", "ps"))
    k = torch.empty((T, M, nkv, dh), device=DEV).normal_(generator=g) * _channels(c, g)
    v = torch.empty((T, M, nkv, dh), device=DEV).normal_(generator=g) * 0.3
    # runs of consecutive tokens, each from a slot of its own on, in pages in any order
    r = np.random.Generator(np.random.PCG64(seed))
    run, slots = c["run"], []
    per = (run + 2 * ps - 2) // ps                                                   # pages of a run, wherever in its first page it begins
    runs = (M + run - 1) // run
    order = r.permutation(runs * per + 2)
    for i in range(runs):
        at = np.arange(min(run, M - i * run)) + int(r.integers(ps))
        slots.append(order[i * per + at // ps] * ps + at % ps)
    slots = np.concatenate(slots).astype(np.int64)
    slots[r.random(M) < c["skip"]] = -1
    pool = torch.randint(0, 120, (T, len(order), nkv, ps // 16, _block_bytes(dh)), dtype=torch.uint8, device=DEV, generator=g)
    s = dict(c, k=k.bfloat16().view(T, M, -1), v=v.bfloat16().view(T, M, -1), pool=pool, slots=torch.from_numpy(slots).to(DEV))
    if c["values"]:
        s.update(k_out=torch.zeros_like(s["k"]), v_out=torch.zeros_like(s["v"]))
    return s


def _pool(c, pages, g):
    """A layer's slabs uint8 [T, pages, nkv, ps / 16, bytes] of K and V as a model leaves them, quantised."""
    size, scale = pages * c["nkv"] * (c["ps"] // 16), _channels(c, g)
    wide = scale.repeat_interleave(c["ps"] // 16, 0).repeat(pages, 1)[:, None]
    out = []
    for _ in range(c["T"]):
        k = torch.empty((size, 16, c["dh"]), device=DEV).normal_(generator=g) * wide
        v = torch.empty((size, 16, c["dh"]), device=DEV).normal_(generator=g) * 0.3
        out.append(_pack(*_quantise(k), *_quantise(v)).view(pages, c["nkv"], c["ps"] // 16, -1))
    return torch.stack(out)


def _table(lens, ps, pages, seed):
    """Block table int32 [B, columns] of sequences in pages in any order."""
    used = [(n + ps - 1) // ps for n in lens]
    order = np.random.Generator(np.random.PCG64(seed)).permutation(pages)
    bt = np.zeros((len(lens), max(used)), np.int32)
    at = 0
    for b, n in enumerate(used):
        bt[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(bt).to(DEV)


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _prepare_read(c, seed, g):
    kv = _lens(c)[1]
    pages = sum((n + c["ps"] - 1) // c["ps"] for n in kv) + 2
    opages = sum((n + c["ops"] - 1) // c["ops"] for n in kv) + 1
    return dict(c, pool=_pool(c, pages, g), bt=_table(kv, c["ps"], pages, seed), kv_len=_ints(kv), keys=sum(kv),
                out=torch.zeros((c["T"], opages, 2, c["nkv"], c["ops"], c["dh"]), dtype=torch.bfloat16, device=DEV),
                obt=_table(kv, c["ops"], opages, seed + 1))


def _prepare_attn(c, seed, g):
    q_len, kv = _lens(c)
    pages = sum((n + c["ps"] - 1) // c["ps"] for n in kv) + 2
    q = torch.empty((c["T"], sum(q_len), c["nq"] * c["dh"]), device=DEV).normal_(generator=g)
    s = dict(c, pool=_pool(c, pages, g), bt=_table(kv, c["ps"], pages, seed), kv_len=_ints(kv), q=q.bfloat16(), q_max=max(q_len), rows=sum(q_len),
             q_len=None if c["q"] == "one" else _ints(q_len))
    s["out"] = torch.zeros_like(s["q"])
    return s


# ---------------------------------------------------------------------------------------------- one pass


def run(s):
    if own:
        from paper_2602_07306_b200 import pt
        shape = dict(nkv=s["nkv"], dh=s["dh"], ps=s["ps"])
        if s["op"] == "write":
            pt.kernel_kv_write_e2m1(s["k"], s["v"], s["pool"], s["slots"], k_out=s.get("k_out"), v_out=s.get("v_out"), **shape)
            return _written(s)
        if s["op"] == "read":
            out, _ = pt.kernel_kv_read_e2m1(s["pool"], s["bt"], s["kv_len"], s["out"], s["obt"], **shape)
            return out
        if "scratch" not in s:
            s["scratch"] = pt.attn_e2m1_scratch(s["T"], s["nq"], s["nkv"], s["dh"], DEV)
        out, _ = pt.kernel_attn_e2m1(s["q"], s["pool"], s["bt"], s["kv_len"], s["q_len"], nq=s["nq"], out=s["out"], scratch=s["scratch"], **shape)
        return out
    return {"write": _write, "read": _read, "attn": _attn}[s["op"]](s)


def _written(s):
    return (s["k_out"], s["v_out"], s["pool"]) if s["values"] else s["pool"]


def _offsets(dh):
    """Place of every code and scale in a block: (byte, shift) [16, dh] of K and V, byte [16, dh / 32] of their scales."""
    s, d = torch.arange(16, device=DEV)[:, None], torch.arange(dh, device=DEV)
    group = torch.arange(dh // 32, device=DEV)
    k = (s % 2 * 8 + s // 2) * (dh // 2) + d % 32 // 8 * (dh // 8) + d // 32 * 4 + d % 8 // 2
    q, i, at = s // 4, s % 4, d // 32 * 2 + d % 4 // 2
    piece = d % 32 // 4 * 4 + q
    v = (i // 2 * 512 + piece * 16 + i % 2 * 8 if dh == 128 else piece * 16 + i * 4) + at
    return k, 8 * dh + s * (dh // 32) + group, 8 * dh + dh // 2 + v, 16 * dh + dh // 2 + q * (dh // 8) + group * 4 + i, (d % 2 * 4).expand(16, dh)


def _write(s):
    T, M, nkv, dh, ps = (s[a] for a in ("T", "M", "nkv", "dh", "ps"))
    (kc, ks), (vc, vs) = (_quantise(s[a].float().view(T, M, nkv, dh)) for a in ("k", "v"))
    if s["values"]:
        s["k_out"].copy_(_values(kc, ks).view(T, M, -1))
        s["v_out"].copy_(_values(vc, vs).view(T, M, -1))
    kept = s["slots"] >= 0
    slot = s["slots"].clamp(min=0)
    pool = s["pool"]
    flat = pool.view(-1)
    # first byte of the block of every (track, row, head)
    size, heads = pool.shape[-1], torch.arange(nkv, device=DEV)
    block = ((torch.arange(T, device=DEV)[:, None, None] * pool.shape[1] + (slot // ps)[:, None]) * nkv + heads) * (ps // 16) + (slot % ps // 16)[:, None]
    kat, ksat, vat, vsat, _ = _offsets(dh)
    put = lambda at, x: flat.index_put_(((block[..., None] * size + at[slot % 16][:, None])[:, kept],), x[:, kept])    # noqa: E731
    put(kat[:, ::2], kc[..., ::2] | kc[..., 1::2] << 4)
    put(ksat, ks)
    put(vat[:, ::2], vc[..., ::2] | vc[..., 1::2] << 4)
    put(vsat, vs)
    return _written(s)


def _tokens(s):
    """K and V of every page, float32 [T, pages, nkv, ps, dh] each."""
    return (a.reshape(*a.shape[:3], -1, a.shape[-1]) for a in _unpack(s["pool"], s["dh"]))


def _read(s):
    ps, ops, out = s["ps"], s["ops"], s["out"]
    end = torch.cumsum(s["kv_len"].long(), 0)
    key = torch.arange(s["keys"], device=DEV)
    b = torch.searchsorted(end, key, right=True)
    pos = key - (end - s["kv_len"])[b]
    page, to = s["bt"][b, pos // ps].long(), s["obt"][b, pos // ops].long()
    for i, x in enumerate(_tokens(s)):
        out[:, to, i, :, pos % ops] = x[:, page, :, pos % ps].to(out.dtype)
    return out


def _attn(s):
    T, B, nq, nkv, dh, S = s["T"], s["B"], s["nq"], s["nkv"], s["dh"], s["q_max"]
    G = nq // nkv
    kv_len = s["kv_len"].long()
    q_len = torch.ones_like(kv_len) if s["q_len"] is None else s["q_len"].long()
    row = torch.arange(s["rows"], device=DEV)
    end = torch.cumsum(q_len, 0)
    b = torch.searchsorted(end, row, right=True)
    at = row - (end - q_len)[b]
    q = torch.zeros((T, B, S, nkv, G, dh), dtype=torch.float32, device=DEV)
    q[:, b, at] = s["q"].float().view(T, s["rows"], nkv, G, dh)
    k, v = (x[:, s["bt"].long()].transpose(2, 3).reshape(T, B, nkv, -1, dh) for x in _tokens(s))
    score = torch.matmul(q.permute(0, 1, 3, 4, 2, 5).reshape(T, B, nkv, G * S, dh), k.transpose(-1, -2)).view(T, B, nkv, G, S, -1) / math.sqrt(dh)
    key = torch.arange(score.shape[-1], device=DEV)
    pos = (kv_len - q_len)[:, None] + torch.arange(S, device=DEV)                    # [B, S]
    seen = (key <= pos[..., None]) & (key < kv_len[:, None, None])                   # [B, S, K]
    score.masked_fill_(~seen[None, :, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(T, B, nkv, G * S, -1), v).view(T, B, nkv, G, S, dh) / total
    s["out"].copy_(o.permute(0, 1, 4, 2, 3, 5)[:, b, at].reshape(T, s["rows"], nq * dh))
    return s["out"]


# ---------------------------------------------------------------------------------------------- what a pass needs


def work(c):
    vec = c["dh"] // 2 + c["dh"] // 32                                               # bytes of a cached vector
    if c["op"] == "write":
        n = 2.0 * c["T"] * c["M"] * c["nkv"]
        return {"bytes": n * (2 * c["dh"] + (1 - c["skip"]) * vec + (2 * c["dh"] if c["values"] else 0)) + 8 * c["M"], "flops": 0.0}
    q_len, kv = _lens(c)
    if c["op"] == "read":
        return {"bytes": 2.0 * c["T"] * c["nkv"] * sum(kv) * (vec + 2 * c["dh"]), "flops": 0.0}
    seen = sum(q * (k - q) + q * (q + 1) // 2 for q, k in zip(q_len, kv))
    read = sum(k for q, k in zip(q_len, kv) if q)
    return {"bytes": 2.0 * c["T"] * (c["nkv"] * read * vec + 2 * c["nq"] * sum(q_len) * c["dh"]), "flops": 4.0 * c["T"] * c["nq"] * c["dh"] * seen}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits


def _exact_rounded(x):
    """Values float64 of x [..., dh] after a way through the cache: the nearest of each group's sixteen multiples of its scale."""
    s = torch.tensor(sorted([m * 2.0 ** -17 for m in range(8)] + [(8 + m) * 2.0 ** (e - 18) for e in range(1, 31) for m in range(8)])[:248], dtype=torch.float64, device=DEV)
    x = x.double()
    g = x.reshape(*x.shape[:-1], -1, 32)
    fits = g.abs().amax(-1, keepdim=True) <= 6 * s
    scale = s[torch.where(fits.any(-1), fits.int().argmax(-1), 247)][..., None]
    y = torch.where(scale > 0, g / scale, 0.0)
    near, best = torch.zeros_like(y), torch.full_like(y, math.inf)
    for m in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):                               # the even codes first: they win a tie
        far = (y.abs() - m).abs()
        near, best = torch.where(far < best, m, near), torch.minimum(far, best)
    return (near * y.sign() * scale).view(x.shape)


def _exact_token(flat, at, slot, page, s):
    """K and V float64 [tokens, dh] of one track and head from the bytes of its blocks: `page` and `slot` of every token."""
    kat, ksat, vat, vsat, shift = at
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=DEV) / 2
    rows = flat[page, slot // 16]                                                    # [tokens, bytes]
    i = slot % 16
    out = []
    for code, scale in ((kat, ksat), (vat, vsat)):
        c = (torch.gather(rows, 1, code[i]) >> shift[i].to(torch.uint8)) & 15
        b = torch.gather(rows, 1, scale[i]).long()
        sc = torch.where(b < 8, b.double(), (8 + b % 8).double() * torch.exp2((b // 8 - 1).double())) * 2.0 ** -17
        out.append(grid[(c & 7).long()] * torch.where(c > 7, -1.0, 1.0).double() * sc.repeat_interleave(32, 1))
    return out


def exact(case, seed):
    c = case
    if c["op"] == "write":
        if not c["values"]:
            return None
        s = prepare(c, seed)
        return *(_exact_rounded(s[a].view(c["T"], c["M"], c["nkv"], c["dh"])).view(s[a].shape) for a in ("k", "v")), None
    q_len, kv = _lens(c)
    s = prepare(c, seed)
    at = _offsets(c["dh"])
    if c["op"] == "read":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        for b, n in enumerate(kv):
            pos = torch.arange(n, device=DEV)
            page, to = s["bt"][b, pos // c["ps"]].long(), s["obt"][b, pos // c["ops"]].long()
            for t in range(c["T"]):
                for h in range(c["nkv"]):
                    for i, x in enumerate(_exact_token(s["pool"][t, :, h], at, pos % c["ps"], page, s)):
                        out[t, to, i, h, pos % c["ops"]] = x
        return out
    if c["T"] * c["nkv"] * c["B"] > 5000:
        return None
    G, dh = c["nq"] // c["nkv"], c["dh"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for b, (S, n) in enumerate(zip(q_len, kv)):
        pos = torch.arange(n, device=DEV)
        page = s["bt"][b, pos // c["ps"]].long()
        hidden = pos > (n - S + torch.arange(S, device=DEV))[:, None]
        for t in range(c["T"] if S else 0):
            for h in range(c["nkv"]):
                k, v = _exact_token(s["pool"][t, :, h], at, pos % c["ps"], page, s)
                q = s["q"][t, row:row + S].double().view(S, c["nq"], dh)[:, h * G:(h + 1) * G]
                a = torch.einsum("sgd,kd->gsk", q, k) * dh ** -0.5
                p = torch.softmax(a.masked_fill(hidden, -math.inf), -1)
                out[t, row:row + S].view(S, c["nq"], dh)[:, h * G:(h + 1) * G] = torch.einsum("gsk,kd->sgd", p, v)
        row += S
    return out
