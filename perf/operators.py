"""Workloads of the serving operators around one Parallel Track forward pass, with their plain forms.

Three operators that a server needs between two forward passes of a batch that changes from step to step:

  chunk   attention of a ragged chunk of new tokens per sequence over the paged KV cache of one layer
          (q_len[b] new tokens of sequence b, their K and V already cached; causal inside the chunk)
  copy    copies of whole cache pages inside a pool, over every (track, layer) slab at once
  sample  one token per row of logits under temperature, top-k, top-p and min-p, from given random numbers

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
        # one user's four speculated tokens against a short context, the head layout of the small bf16 workload
        dict(name="chunk_4_tokens_short", op="chunk", T=4, B=1, nq=8, nkv=8, dh=64, ps=16, q="fixed", q_hi=4, kv_lo=301, kv_hi=301, lens=1),
        # speculated tokens of eight users at the decode workload's shape (8 tracks, 8 heads, 2k context)
        dict(name="chunk_verify_8x2k", op="chunk", T=8, B=8, nq=8, nkv=8, dh=128, ps=16, q="ragged", q_hi=8, kv_lo=1800, kv_hi=2300, lens=2),
        # few users with long contexts, grouped heads: every key range has to be split over the machine
        dict(name="chunk_verify_4x30k", op="chunk", T=4, B=4, nq=16, nkv=4, dh=128, ps=32, q="fixed", q_hi=5, kv_lo=9000, kv_hi=31000, lens=3),
        # a step of continuous batching: 27 sequences decode one token while another's prompt advances by 777
        dict(name="chunk_mixed_28", op="chunk", T=4, B=28, nq=16, nkv=4, dh=128, ps=16, q="mixed", q_hi=777, kv_lo=800, kv_hi=4096, lens=4),
        # one 2048-token chunk of a long prompt, 8 query heads on one KV head (the paper's head layout)
        dict(name="chunk_2048_of_32k", op="chunk", T=2, B=1, nq=8, nkv=1, dh=128, ps=16, q="fixed", q_hi=2048, kv_lo=32000, kv_hi=32000, lens=5),
        # a forked sequence of a small model writes to its shared last page
        dict(name="copy_1_page_small", op="copy", T=4, L=8, nkv=8, dh=64, ps=16, pages=64, n=1, fmt="bf16", shared=False),
        # one prompt answered 24 times: every answer's last page is made its own (decode workload's cache)
        dict(name="copy_24_forks", op="copy", T=8, L=32, nkv=8, dh=128, ps=16, pages=96, n=24, fmt="bf16", shared=True),
        # compaction of an 8-bit cache: half of its pages move to the front
        dict(name="copy_compact_8bit", op="copy", T=4, L=48, nkv=4, dh=128, ps=32, pages=301, n=150, fmt="e4m3", shared=False),
        # one row of the default vocabulary with the usual filters: latency
        dict(name="sample_1x32000", op="sample", n=1, V=32000, mode="all", scale=2.5, fmt="f32", pad=0, masked=0.0),
        # a batch with an odd vocabulary, half of it masked by a grammar, every row with its own settings
        dict(name="sample_17x50021_mixed", op="sample", n=17, V=50021, mode="mixed", scale=3.0, fmt="f32", pad=3, masked=0.5),
        # nucleus sampling of a decode batch over a large vocabulary
        dict(name="sample_64x128000_top_p", op="sample", n=64, V=128000, mode="top_p", scale=2.0, fmt="f32", pad=0, masked=0.0),
        # the largest decode batch, mixed settings: the logits are a gigabyte-scale stream
        dict(name="sample_1000x128000_mixed", op="sample", n=1000, V=128000, mode="mixed", scale=2.5, fmt="f32", pad=0, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "copy", "sample", "sample"])
    if op == "chunk":
        nkv, g = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8])
        kind = rng.choice(["fixed", "ragged", "mixed"])
        c = dict(op=op, T=rng.choice([1, 2, 3, 4, 8]), B=_log(rng, 1, 40), nq=nkv * g, nkv=nkv, dh=rng.choice([64, 128, 128]), ps=rng.choice([16, 32, 48, 64]),
                 q=kind, q_hi=_log(rng, 1, 16) if rng.random() < 0.6 else _log(rng, 16, 1500), kv_lo=0, kv_hi=_log(rng, 40, 30000), lens=rng.randrange(1 << 20))
        c["kv_hi"] = max(c["kv_hi"], c["q_hi"] + 1)
        c["kv_lo"] = rng.randint(1, c["kv_hi"])
        # no more than the largest listed case: scores of the plain form, and bytes
        while c["B"] > 1 and (c["T"] * c["B"] * c["nq"] * c["q_hi"] * c["kv_hi"] > 1.0e9 or c["T"] * c["B"] * c["nkv"] * c["kv_hi"] * c["dh"] > 4.0e8):
            c["B"] = (c["B"] + 1) // 2
        while c["T"] * c["B"] * c["nq"] * c["q_hi"] * c["kv_hi"] > 1.0e9 or c["T"] * c["B"] * c["nkv"] * c["kv_hi"] * c["dh"] > 4.0e8:
            c["kv_hi"] = max(40, c["kv_hi"] * 2 // 3)
            c["kv_lo"] = min(c["kv_lo"], c["kv_hi"])
            c["q_hi"] = max(1, min(c["q_hi"] * 2 // 3, c["kv_hi"] - 1))
        return c
    if op == "copy":
        fmt = rng.choice(["bf16", "bf16", "e4m3"])
        c = dict(op=op, T=rng.choice([1, 2, 4, 8]), L=_log(rng, 2, 48), nkv=rng.choice([1, 2, 4, 8]), dh=128 if fmt == "e4m3" else rng.choice([32, 64, 128]),
                 ps=rng.choice([16, 32, 48, 64] if fmt == "e4m3" else [8, 16, 24, 32, 64]), pages=0, n=_log(rng, 1, 200), fmt=fmt, shared=rng.random() < 0.4)
        while c["n"] > 1 and _page_bytes(c) * c["T"] * c["L"] * c["n"] > 600e6:
            c["n"] = (c["n"] + 1) // 2
        c["pages"] = 2 * c["n"] + rng.randint(1, 40)
        return c
    V = rng.choice([_log(rng, 300, 200000), _log(rng, 300, 200000), 32000])
    n = _log(rng, 1, max(1, min(1000, int(6e7 / V))))
    return dict(op=op, n=n, V=V, mode=rng.choice(["all", "mixed", "top_k", "top_p", "min_p", "plain"]), scale=rng.choice([1.0, 2.0, 3.0, 5.0]),
                fmt=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0, 0, 1, 5, 64]), masked=rng.choice([0.0, 0.0, 0.3, 0.9]))


def _lens(c):
    """New tokens and cached keys of every sequence of a chunk case: plain lists, from the case alone."""
    r = random.Random(c["lens"])
    kv = [r.randint(c["kv_lo"], c["kv_hi"]) for _ in range(c["B"])]
    if c["q"] == "fixed":
        q = [c["q_hi"]] * c["B"]
    elif c["q"] == "ragged":                       # idle sequences among them
        q = [r.randint(0, c["q_hi"]) for _ in range(c["B"])]
    else:                                          # one long chunk among single tokens
        q = [1] * c["B"]
        q[r.randrange(c["B"])] = c["q_hi"]
    q[0] = max(1, q[0])
    return [min(a, b) for a, b in zip(q, kv)], kv


def _page_bytes(c):
    vec = 2 * c["nkv"] * c["ps"]
    return vec * (c["dh"] + 4) if c["fmt"] == "e4m3" else vec * c["dh"] * 2


# ---------------------------------------------------------------------------------------------- inputs


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"chunk": _prepare_chunk, "copy": _prepare_copy, "sample": _prepare_sample}[case["op"]](case, seed, g)


def _prepare_chunk(c, seed, g):
    q_len, kv_len = _lens(c)
    rows, maxp = sum(q_len), max((k + c["ps"] - 1) // c["ps"] for k in kv_len)
    used = [(k + c["ps"] - 1) // c["ps"] for k in kv_len]
    pages = sum(used) + 3
    order = np.random.Generator(np.random.PCG64(seed)).permutation(pages)
    bt = np.zeros((c["B"], maxp), np.int32)
    at = 0
    for b, n in enumerate(used):
        bt[b, :n] = order[at:at + n]
        at += n
    pool = torch.empty((c["T"], pages, 2, c["nkv"], c["ps"], c["dh"]), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    q = torch.empty((c["T"], rows, c["nq"] * c["dh"]), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    return dict(c, q=q * 1.5, pool=pool, bt=torch.from_numpy(bt).to(DEV), out=torch.zeros_like(q),
                q_len=torch.tensor(q_len, dtype=torch.int32, device=DEV), kv_len=torch.tensor(kv_len, dtype=torch.int32, device=DEV),
                q_max=max(q_len), rows=rows)


def _prepare_copy(c, seed, g):
    r = np.random.Generator(np.random.PCG64(seed)).permutation(c["pages"]).astype(np.int32)
    n = c["n"]
    src, dst = (np.full(n, r[0], np.int32) if c["shared"] else r[:n].copy()), r[n:2 * n].copy()
    shape = (c["T"], c["L"], c["pages"], 2, c["nkv"], c["ps"])
    s = dict(c, src=src, dst=dst, src_d=torch.from_numpy(src).to(DEV).long(), dst_d=torch.from_numpy(dst).to(DEV).long())
    if c["fmt"] == "e4m3":
        s["pool"] = torch.randint(0, 126, shape + (c["dh"],), dtype=torch.uint8, device=DEV, generator=g)
        s["scales"] = torch.exp2(torch.randint(-12, 3, shape, device=DEV, generator=g).float())
    else:
        s["pool"] = torch.empty(shape + (c["dh"],), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    return s


def _prepare_sample(c, seed, g):
    n, V = c["n"], c["V"]
    dt = torch.float32 if c["fmt"] == "f32" else torch.bfloat16
    full = torch.empty((n, V + c["pad"]), dtype=torch.float32, device=DEV).normal_(generator=g).mul_(c["scale"])
    if c["masked"]:
        full.masked_fill_(torch.rand(full.shape, device=DEV, generator=g) < c["masked"], -math.inf)
    logits = full.to(dt)[:, :V]
    r = np.random.Generator(np.random.PCG64(seed))
    pick = lambda a: r.choice(np.array(a), n)                                       # noqa: E731
    off = dict(t=np.full(n, 1.0), k=np.zeros(n, np.int64), p=np.ones(n), m=np.zeros(n))
    if c["mode"] == "all":
        off.update(t=np.full(n, 0.8), k=np.full(n, 50), p=np.full(n, 0.95), m=np.full(n, 0.02))
    elif c["mode"] == "mixed":
        off.update(t=pick([0.0, 0.3, 0.7, 1.0, 1.3]), k=pick([0, 1, 20, 50, 1000]), p=pick([1.0, 0.8, 0.95, 0.999]), m=pick([0.0, 0.05, 0.2]))
    elif c["mode"] == "top_k":
        off.update(t=np.full(n, 0.9), k=pick([1, 5, 40, 200]))
    elif c["mode"] == "top_p":
        off.update(t=np.full(n, 1.0), p=pick([0.5, 0.9, 0.95]))
    elif c["mode"] == "min_p":
        off.update(t=np.full(n, 1.2), m=pick([0.02, 0.1]))
    f = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV)                    # noqa: E731
    return dict(c, logits=logits, temperature=f(off["t"]), top_k=torch.from_numpy(off["k"].astype(np.int32)).to(DEV), top_p=f(off["p"]), min_p=f(off["m"]),
                u=torch.rand(n, dtype=torch.float32, device=DEV, generator=g), token=torch.empty(n, dtype=torch.int32, device=DEV),
                prob=torch.empty(n, dtype=torch.float32, device=DEV))


# ---------------------------------------------------------------------------------------------- one pass


def run(s):
    if own:
        from paper_2602_07306_b200 import pt
        if s["op"] == "chunk":
            if "scratch" not in s:
                s["scratch"] = pt.chunk_attn_scratch(s["T"], s["B"], s["nq"], s["dh"], DEV)
            out, _ = pt.kernel_chunk_attn(s["q"], s["pool"], s["bt"], s["q_len"], s["kv_len"], nq=s["nq"], nkv=s["nkv"], dh=s["dh"], ps=s["ps"],
                                          out=s["out"], scratch=s["scratch"])
            return out
        if s["op"] == "copy":
            pt.kernel_kv_copy_pages(s["pool"], s["src"], s["dst"], scales=s.get("scales"))
            return _copied(s)
        return pt.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], out=s["token"], prob=s["prob"])
    return {"chunk": _chunk, "copy": _copy, "sample": _sample}[s["op"]](s)


def _chunk(s):
    T, B, nq, nkv, dh, S = s["T"], s["B"], s["nq"], s["nkv"], s["dh"], s["q_max"]
    G = nq // nkv
    q_len, kv_len = s["q_len"].long(), s["kv_len"].long()
    row = torch.arange(s["rows"], device=DEV)
    end = torch.cumsum(q_len, 0)
    b = torch.searchsorted(end, row, right=True)
    at = row - (end - q_len)[b]
    q = torch.zeros((T, B, S, nkv, G, dh), dtype=torch.float32, device=DEV)
    q[:, b, at] = s["q"].float().view(T, s["rows"], nkv, G, dh)
    kv = s["pool"][:, s["bt"].long()].float()                                        # [T, B, maxp, 2, nkv, ps, dh]
    k, v = (kv[:, :, :, i].transpose(2, 3).reshape(T, B, nkv, -1, dh) for i in (0, 1))
    del kv
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


def _copied(s):
    return (s["pool"].view(torch.float8_e4m3fn), s["scales"]) if s["fmt"] == "e4m3" else s["pool"]


def _copy(s):
    pool = s["pool"].view(s["T"] * s["L"], s["pages"], -1)
    pool[:, s["dst_d"]] = pool[:, s["src_d"]]
    if s["fmt"] == "e4m3":
        scales = s["scales"].view(s["T"] * s["L"], s["pages"], -1)
        scales[:, s["dst_d"]] = scales[:, s["src_d"]]
    return _copied(s)


def _sample(s):
    # weights and their sums in 64 bits: a cumulative sum decides which token a random number falls on
    x = s["logits"].double()
    n, V = x.shape
    greedy = s["temperature"] <= 0
    t = torch.where(greedy, 1.0, s["temperature"].double())[:, None]
    k = torch.where(greedy, 1, torch.where((s["top_k"] > 0) & (s["top_k"] < V), s["top_k"], V).long())[:, None]
    x, at = torch.sort(x, dim=1, descending=True, stable=True)                       # equal logits: the lower index first
    w = torch.exp((x - x[:, :1]) / t)
    w = torch.where(torch.arange(V, device=DEV) < k, w, 0.0)
    before = torch.cumsum(w, 1)
    keep = (before - w < s["top_p"].double()[:, None] * before[:, -1:]) | (s["top_p"][:, None] >= 1)
    w = torch.where(keep & (w >= s["min_p"].double()[:, None]), w, 0.0)
    w = torch.zeros_like(w).scatter_(1, at, w)                                       # back in the vocabulary's order
    upto = torch.cumsum(w, 1)
    total = upto[:, -1:]
    token = torch.searchsorted(upto, s["u"].double()[:, None] * total, right=True).clamp_(max=V - 1)
    s["token"].copy_(token[:, 0])
    s["prob"].copy_((torch.gather(w, 1, token) / total)[:, 0])
    return s["token"], s["prob"]


# ---------------------------------------------------------------------------------------------- what a pass needs


def work(c):
    if c["op"] == "chunk":
        q_len, kv_len = _lens(c)
        seen = sum(q * (k - q) + q * (q + 1) // 2 for q, k in zip(q_len, kv_len))
        read = sum(k for q, k in zip(q_len, kv_len) if q)
        return {"bytes": 2.0 * c["T"] * c["dh"] * (2 * c["nkv"] * read + 2 * c["nq"] * sum(q_len)), "flops": 4.0 * c["T"] * c["nq"] * c["dh"] * seen}
    if c["op"] == "copy":
        return {"bytes": float(c["T"] * c["L"] * _page_bytes(c)) * (c["n"] + (1 if c["shared"] else c["n"])), "flops": 0.0}
    return {"bytes": float(c["n"]) * (c["V"] * (4 if c["fmt"] == "f32" else 2) + 28), "flops": 0.0}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "chunk":
        q_len, kv_len = _lens(case)
        nkv, G, dh, ps = case["nkv"], case["nq"] // case["nkv"], case["dh"], case["ps"]
        out = torch.zeros((case["T"], sum(q_len), case["nq"] * dh), dtype=torch.float64, device=DEV)
        row = 0
        for b, (S, K) in enumerate(zip(q_len, kv_len)):
            table = s["bt"][b, :(K + ps - 1) // ps].long()
            causal = torch.ones((S, K), dtype=torch.bool, device=DEV).tril(K - S)
            for t in range(case["T"] if S else 0):
                blocks = s["pool"][t, table].double()                                # [pages, 2, nkv, ps, dh]
                for h in range(nkv):
                    k, v = (blocks[:, i, h].reshape(-1, dh)[:K] for i in (0, 1))
                    for j in range(h * G, h * G + G):
                        a = s["q"][t, row:row + S, j * dh:(j + 1) * dh].double() @ k.T * dh ** -0.5
                        p = torch.softmax(torch.where(causal, a, torch.full_like(a, -math.inf)), dim=-1)
                        out[t, row:row + S, j * dh:(j + 1) * dh] = p @ v
            row += S
        return out
    if case["op"] == "copy":
        values = s["pool"].view(torch.float8_e4m3fn) if case["fmt"] == "e4m3" else s["pool"]
        frm = torch.arange(case["pages"], device=DEV)
        frm[s["dst_d"]] = s["src_d"]                                                 # every page of the result, and whose values it holds
        moved = values.double().index_select(2, frm)
        return (moved, s["scales"].double().index_select(2, frm)) if case["fmt"] == "e4m3" else moved
    if case["n"] * case["V"] > 2e8:
        return None
    token, prob = [], []
    for x, u, t, k, p, m in zip(s["logits"], *(s[a].tolist() for a in ("u", "temperature", "top_k", "top_p", "min_p"))):
        x = x.double()
        if t <= 0:
            token.append(int((x == x.max()).nonzero()[0, 0]))
            prob.append(1.0)
            continue
        left = torch.exp((x - x.max()) / t)
        order = torch.argsort(x, descending=True, stable=True)
        left = left[order]
        kept = k if 0 < k < len(x) else len(x)
        if p < 1:
            c = torch.cumsum(left[:kept], 0)
            kept = int((c < p * c[-1]).sum()) + 1
        kept = min(kept, max(1, int((left >= m).sum())))
        ids = order[:kept].sort().values
        pr = torch.exp((x[ids] - x.max()) / t)
        pr = pr / pr.sum()
        j = min(int((torch.cumsum(pr, 0) <= u).sum()), kept - 1)
        token.append(int(ids[j]))
        prob.append(float(pr[j]))
    return torch.tensor(token, dtype=torch.int32), torch.tensor(prob, dtype=torch.float64)
