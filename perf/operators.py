"""Performance cases of the operators that read a user's history in order: rotary positions with per-head norms
(dlrm_qk_rope_*), attention over the sequences of a CSR batch (dlrm_seq_attn_*), and attention of one new item over a paged
cache of the history (dlrm_cache_attn).

A case's "op" is what one pass does:
  rope_train : norms and rotation of queries and keys, then their backward from given gradients
  append     : norms and rotation of new items' queries and keys, keys and values stored in the pages of the cache
  attn       : attention forward over ragged sequences (scoring)
  attn_train : attention forward and backward
  cache      : one new query for each user over the paged cache
Lengths of the sequences of a case are spread evenly over [lo, hi] and shuffled by the seed, so the work of a case is
the same for every seed.  Sizes are those of workloads/gen.py and of the tests (batches 64, 128, 500, 1999, 2048; histories up
to 200 items; widths 16 to 128) and generic ones for long histories."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def _rope(name, op, B, lo, hi, Hq, Hk, d, dtype, rot, layout, norm=True, stretch=1.0, page=16, start=(0, 0)):
    """start: new items come after start[0]..start[1] items that the user's cache holds already."""
    c = dict(name=name, op=op, B=B, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, dtype=dtype, rot=rot, layout=layout, norm=norm,
             stretch=stretch, page=page, start_lo=start[0], start_hi=start[1])
    if not name:
        del c["name"]
    return c


def _attn(name, op, B, q, k, Hq, Hk, d, dtype, causal=True, prefix=False, slopes=False, cap=0.0):
    """q, k: (lo, hi) lengths; k None: every item attends over its own sequence."""
    c = dict(name=name, op=op, B=B, lo=q[0], hi=q[1], self=k is None, klo=(k or q)[0], khi=(k or q)[1], Hq=Hq, Hk=Hk, d=d,
             dtype=dtype, causal=causal, prefix=prefix, slopes=slopes, cap=cap)
    if not name:
        del c["name"]
    return c


def _cache(name, B, lo, hi, Hq, Hk, d, dtype, page, slopes=False, cap=0.0):
    c = dict(name=name, op="cache", B=B, lo=lo, hi=hi, Hq=Hq, Hk=Hk, d=d, dtype=dtype, page=page, slopes=slopes, cap=cap)
    if not name:
        del c["name"]
    return c


def listed():
    return [
        # one new item of each of 64 users being served: its key and value go into the cache (latency of one launch)
        _rope("append_serve_b64", "append", 64, 1, 1, 8, 2, 64, "bf16", 64, "half", page=64, start=(1, 2000)),
        # first visit of 500 users: their histories go into the cache at once, half of each head rotated
        _rope("append_prompts_f16", "append", 500, 1, 200, 8, 8, 64, "f16", 32, "interleaved"),
        # training on ordinary histories (batch 2048, up to 200 items) in the framework's own fp32
        _rope("rope_train_f32", "rope_train", 2048, 1, 200, 4, 4, 64, "f32", 64, "interleaved"),
        # long histories, positions stretched, few key heads
        _rope("rope_train_long", "rope_train", 8, 2048, 16384, 16, 4, 128, "bf16", 128, "half", stretch=4.0),
        # the smallest training batch: 128 users with next to no history, some with none
        _attn("attn_train_tiny", "attn_train", 128, (0, 20), None, 2, 2, 16, "f32"),
        # ordinary histories in bf16, older items weigh less
        _attn("attn_train_history", "attn_train", 2048, (1, 200), None, 4, 4, 64, "bf16", slopes=True),
        # long histories, capped scores, four query heads to a key head: the largest
        _attn("attn_train_long", "attn_train", 8, (2048, 4096), None, 16, 4, 128, "bf16", cap=30.0),
        # odd sizes in fp32, the first quarter of a history (profile items) seen by all of it
        _attn("attn_train_odd_f32", "attn_train", 13, (1, 1999), None, 6, 3, 72, "f32", prefix=True),
        # candidates scored against histories, some of them empty; two key heads, an odd width
        _attn("attn_candidates_f16", "attn", 500, (1, 40), (0, 1000), 8, 2, 40, "f16", causal=False),
        # 64 users with short histories in fp32: latency
        _cache("cache_serve_f32", 64, 1, 200, 4, 4, 64, "f32", 16),
        # one user with a very long history: the length is all there is to split
        _cache("cache_one_long", 1, 131072, 131072, 16, 4, 128, "bf16", 64),
        # a full serving batch of mixed lengths, capped, older items weigh less: the largest of its kind
        _cache("cache_batch_mixed", 256, 1, 8192, 16, 4, 128, "bf16", 32, slopes=True, cap=50.0),
    ]


def draw(rng):
    """Another case of the same ranges: any operator, batch, lengths, heads, width, type and mask, at most as much work as
    the largest listed case of its kind."""
    logu = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    while True:
        op = rng.choice(["append", "rope_train", "attn", "attn_train", "attn_train", "cache", "cache"])
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        Hk = rng.choice([1, 2, 3, 4, 8])
        Hq = Hk * rng.choice([1, 1, 2, 4, 5, 8])
        d = 8 * logu(1, 16)
        B = logu(1, 2048)
        if op in ("append", "rope_train"):
            hi = logu(1, 16384)
            c = _rope("", op, B, rng.choice([1, max(1, hi // 2), hi]), hi, Hq, Hk, d, dtype, 2 * rng.randint(1, d // 2),
                      rng.choice(["half", "interleaved"]), norm=rng.random() < 0.7, stretch=rng.choice([1.0, 4.0]),
                      page=2 ** rng.randint(3, 7), start=(0, logu(1, 2000)) if op == "append" else (0, 0))
            if int(_lengths(c).sum()) * (Hq + 2 * Hk) * d <= 8 * 16384 * 24 * 128 and (op != "append" or B * _cache_cols(c) * c["page"] * Hk * d <= 4e8):
                return c
        elif op == "cache":
            hi = logu(1, 131072)
            c = _cache("", B, rng.choice([0, 1, hi // 2, hi]), hi, Hq, Hk, d, dtype, 2 ** rng.randint(3, 7),
                       slopes=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 30.0]))
            if B * hi * Hk * d <= 256 * 8192 * 4 * 128 and B * hi * Hq <= 256 * 8192 * 16:
                return c
        else:
            hi = logu(1, 4096)
            alone = rng.random() < 0.7
            khi = hi if alone else logu(1, 4096)
            causal = rng.random() < 0.7
            c = _attn("", op, B, (rng.choice([0, 1, hi // 2, hi]), hi), None if alone else (rng.choice([0, 1, khi]), khi), Hq, Hk, d, dtype,
                      causal=causal, prefix=causal and rng.random() < 0.3, slopes=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 30.0]))
            if B * Hq * hi * khi <= 8 * 16 * 4096 * 4096 and B * (hi + khi) * Hq * d <= 2048 * 400 * 16 * 128:
                return c


# ---------------------------------------------------------------------------------------------- sizes
def _even(n, lo, hi):
    return np.rint(np.linspace(hi, lo, n)).astype(np.int64)


def _lengths(c):
    return _even(c["B"], c["lo"], c["hi"])


def _cache_cols(c):
    return (c["hi"] + c.get("start_hi", 0) + c["page"] - 1) // c["page"]


def _pairs(c):
    """Visible (query, key) pairs of a case, those of sequences of queries and keys of their own taken at their means."""
    lq, lk = _lengths(c), _even(c["B"], c["klo"], c["khi"])
    if not c["causal"]:
        return float((lq * lk).sum()) if c["self"] else float(lq.sum()) * float(lk.mean())
    if not c["self"]:  # a query sees the keys up to its own place, counted from the end
        nq, nk = float(lq.mean()), float(lk.mean())
        m = min(nq, nk)
        return c["B"] * (m * nk - m * (m - 1) / 2)
    p = lq // 4 if c["prefix"] else 0 * lq  # the first p queries see p keys each
    return float((p * p + (lq * (lq + 1) - p * (p + 1)) / 2).sum())


def work(c):
    e, d, Hq, Hk = DTYPES[c["dtype"]].itemsize, c["d"], c["Hq"], c["Hk"]
    T = int(_lengths(c).sum())
    if c["op"] == "append":
        return {"bytes": T * ((2 * Hq + 4 * Hk) * d * e + 8), "flops": T * (Hq + Hk) * d * 8}
    if c["op"] == "rope_train":
        return {"bytes": T * (Hq + Hk) * d * e * 5, "flops": T * (Hq + Hk) * d * 30}
    if c["op"] == "cache":
        return {"bytes": T * Hk * d * e * 2 + 2 * c["B"] * Hq * d * e, "flops": T * Hq * d * 4}
    Tk = int(_even(c["B"], c["klo"], c["khi"]).sum())
    rows = T * Hq * d * e * 2 + Tk * Hk * d * e * 2
    if c["op"] == "attn":
        return {"bytes": rows + T * Hq * 4, "flops": _pairs(c) * Hq * d * 4}
    return {"bytes": 2 * rows + T * Hq * d * e * 2, "flops": _pairs(c) * Hq * d * 14}


# ---------------------------------------------------------------------------------------------- inputs
def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=DEV)


def _pages(g, B, cols):
    """The pages of B users, in the order in which a pool that has been in use for a while hands them out."""
    return torch.randperm(B * cols, generator=g, device=DEV).to(torch.int32).view(B, cols)


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 32))
    dt, B, Hq, Hk, d = DTYPES[c["dtype"]], c["B"], c["Hq"], c["Hk"], c["d"]
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dt)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=t)
    s = {"c": c}
    lens = rng.permutation(_lengths(c))
    T = int(lens.sum())
    if c["op"] in ("append", "rope_train"):
        # queries, keys and values leave one projection, side by side in a row
        qkv = rand(T, Hq + 2 * Hk, d)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        start = rng.permutation(_even(B, c["start_lo"], c["start_hi"]))
        seqs = np.repeat(np.arange(B), lens)
        s["positions"] = dev(np.arange(T) - np.repeat(_offsets(lens)[:-1], lens) + start[seqs], torch.int32)
        s["inv_freq"] = 10000.0 ** (-torch.arange(c["rot"] // 2, dtype=torch.float32, device=DEV) * 2 / c["rot"]) / c["stretch"]
        s["wq"], s["wk"] = ((1 + 0.1 * torch.randn(2, d, generator=g, device=DEV)).unbind(0)) if c["norm"] else (None, None)
        s["q_out"] = torch.empty(T, Hq, d, dtype=dt, device=DEV)
        if c["op"] == "append":
            s["seqs"] = dev(seqs, torch.int32)
            cols = _cache_cols(c)
            s["table"] = _pages(g, B, cols)
            s["cache_k"] = torch.zeros(B * cols, Hk, c["page"], d, dtype=dt, device=DEV)
            s["cache_v"] = torch.zeros(B * cols, Hk, c["page"], d, dtype=dt, device=DEV)
        else:
            s["dq_out"], s["dk_out"] = rand(T, Hq, d), rand(T, Hk, d)
            s["k_out"] = torch.empty(T, Hk, d, dtype=dt, device=DEV)
            s["dqkv"] = torch.empty(T, Hq + Hk, d, dtype=dt, device=DEV)
            s["dw"] = torch.empty(2, d, dtype=torch.float32, device=DEV) if c["norm"] else None
    elif c["op"] == "cache":
        cols = max(1, _cache_cols(c))
        s["q"] = rand(B, Hq, d)
        s["table"], s["lens"] = _pages(g, B, cols), dev(lens, torch.int32)
        s["cache_k"], s["cache_v"] = rand(B * cols, Hk, c["page"], d), rand(B * cols, Hk, c["page"], d)
        s["slopes"] = _slopes(Hq) if c["slopes"] else None
        s["out"] = torch.empty(B, Hq, d, dtype=dt, device=DEV)
    else:
        klens = lens if c["self"] else rng.permutation(_even(B, c["klo"], c["khi"]))
        Tk = int(klens.sum())
        if c["self"]:
            qkv = rand(T, Hq + 2 * Hk, d)
            s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        else:
            kv = rand(Tk, 2 * Hk, d)
            s["q"], s["k"], s["v"] = rand(T, Hq, d), kv[:, :Hk], kv[:, Hk:]
        s["q_off"], s["k_off"] = dev(_offsets(lens), torch.int64), dev(_offsets(klens), torch.int64)
        s["prefix"] = dev(klens // 4, torch.int32) if c["prefix"] else None
        s["slopes"] = _slopes(Hq) if c["slopes"] else None
        s["out"], s["lse"] = torch.empty(T, Hq, d, dtype=dt, device=DEV), torch.empty(Hq, T, device=DEV)
        s["max_q"], s["max_k"] = int(lens.max()), int(klens.max())
        if c["op"] == "attn_train":
            s["dout"], s["dq"] = rand(T, Hq, d), torch.empty(T, Hq, d, dtype=dt, device=DEV)
            s["dk"], s["dv"] = (torch.empty(Tk, Hk, d, dtype=dt, device=DEV) for _ in range(2))
    if own:
        import paper_1906_00091_amd as hot
        if c["op"] in ("append", "rope_train"):
            s["plan"] = hot.QkRope(s["positions"], Hq, Hk, d, inv_freq=s["inv_freq"], rot=c["rot"],
                                   layout=hot.ROPE_HALF if c["layout"] == "half" else hot.ROPE_INTERLEAVED, wq=s["wq"], wk=s["wk"], eps=EPS)
            if c["op"] == "append":
                s["cache"] = hot.KvCache(s["cache_k"], s["cache_v"], s["table"])
            else:
                s["ws"] = hot.alloc_qk_rope_workspace(s["plan"])
        elif c["op"] == "cache":
            s["cache"] = hot.KvCache(s["cache_k"], s["cache_v"], s["table"])
            s["ws"] = hot.alloc_cache_attn_workspace(s["cache"], Hq, max(1, c["hi"]))
        else:
            s["plan"] = hot.SeqBatch(s["q_off"], s["k_off"], T, Tk, s["max_q"], s["max_k"], causal=c["causal"], prefix=s["prefix"],
                                     slopes=s["slopes"], cap=c["cap"])
            if c["op"] == "attn_train":
                s["ws"] = hot.alloc_seq_attn_workspace(s["plan"], Hq, Hk, d)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)(s, s["c"])


def _own(s, c):
    import paper_1906_00091_amd as hot
    if c["op"] == "append":
        hot.dlrm_qk_rope_append(s["plan"], s["q"], s["k"], s["v"], s["q_out"], s["cache"], s["seqs"])
        return {"q": s["q_out"], "cache_k": s["cache_k"], "cache_v": s["cache_v"]}
    if c["op"] == "rope_train":
        dq, dk = s["dqkv"][:, :c["Hq"]], s["dqkv"][:, c["Hq"]:]
        hot.dlrm_qk_rope_fwd(s["plan"], s["q"], s["k"], s["q_out"], s["k_out"])
        hot.dlrm_qk_rope_bwd(s["plan"], s["q"], s["k"], s["dq_out"], s["dk_out"], dq, dk, *(s["dw"] if c["norm"] else (None, None)), s["ws"])
        return {"q": s["q_out"], "k": s["k_out"], "dq": dq, "dk": dk, **({"dw": s["dw"]} if c["norm"] else {})}
    if c["op"] == "cache":
        hot.dlrm_cache_attn(s["cache"], s["lens"], max(1, c["hi"]), s["q"], s["out"], s["ws"], slopes=s["slopes"], cap=c["cap"])
        return {"out": s["out"]}
    hot.dlrm_seq_attn_fwd(s["plan"], s["q"], s["k"], s["v"], s["out"], s["lse"])
    if c["op"] == "attn":
        return {"out": s["out"]}
    hot.dlrm_seq_attn_bwd(s["plan"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], s["ws"])
    return {"out": s["out"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _turn(x, cos, sin, layout):
    """Rotates the pairs of the first 2 * cos.shape[-1] columns of x [T, H, d]; cos, sin: [T, 1, pairs]."""
    n = cos.shape[-1]
    head, tail = x[..., :2 * n], x[..., 2 * n:]
    a, b = (head[..., :n], head[..., n:]) if layout == "half" else (head[..., 0::2], head[..., 1::2])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.cat(y, -1) if layout == "half" else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, tail], -1)


def _angles(s):
    # in 64 bits: a position of some thousands times a frequency near 1 leaves 32 bits too few digits after the point
    angle = (s["positions"].double()[:, None] * s["inv_freq"].double()).unsqueeze(1)
    return angle.cos().float(), angle.sin().float()


def _normed(x, w):
    """(normed rows without the weight, 1 / root mean square); x itself where there is no norm."""
    x = x.float()
    if w is None:
        return x, None
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _rope_bwd(x, w, dy, cos, sin, layout):
    n, r = _normed(x, w)
    g = _turn(dy.float(), cos, -sin, layout)
    if w is None:
        return g.to(x.dtype), None
    gw = g * w
    return (r * (gw - n * (gw * n).mean(-1, keepdim=True))).to(x.dtype), (g * n).sum((0, 1))


def _padded(x, off, L):
    """Rows of x [T, H, d] by sequence, [B, H, L, d] in fp32, zeros behind a sequence's end; and which are rows."""
    at = torch.arange(L, device=x.device)
    there = at < (off[1:] - off[:-1])[:, None]
    rows = (off[:-1, None] + at).clamp(max=max(0, x.shape[0] - 1))
    y = x.float()[rows] * there[:, :, None, None]
    return y.transpose(1, 2).contiguous(), there


def _softmax(sc, seen):
    sc = sc.masked_fill(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _plain(s, c):
    dt, Hq, Hk, d = DTYPES[c["dtype"]], c["Hq"], c["Hk"], c["d"]
    if c["op"] in ("append", "rope_train"):
        cos, sin = _angles(s)
        heads = ((s["q"], s["wq"]), (s["k"], s["wk"]))
        q, k = (_turn(_normed(x, w)[0] * (1.0 if w is None else w), cos, sin, c["layout"]).to(dt) for x, w in heads)
        if c["op"] == "append":
            p = s["positions"].long()
            page = s["table"][s["seqs"].long(), p // c["page"]].long()
            s["cache_k"][page, :, p % c["page"]] = k
            s["cache_v"][page, :, p % c["page"]] = s["v"]
            return {"q": q, "cache_k": s["cache_k"], "cache_v": s["cache_v"]}
        (dq, dwq), (dk, dwk) = (_rope_bwd(x, w, dy, cos, sin, c["layout"]) for (x, w), dy in zip(heads, (s["dq_out"], s["dk_out"])))
        return {"q": q, "k": k, "dq": dq, "dk": dk, **({"dw": torch.stack([dwq, dwk])} if c["norm"] else {})}

    scale, G, B = 1.0 / math.sqrt(d), Hq // Hk, c["B"]
    if c["op"] == "cache":
        L = s["table"].shape[1] * c["page"]
        k, v = (s[n][s["table"].long()].float().transpose(1, 2).reshape(B, Hk, L, d) for n in ("cache_k", "cache_v"))
        q = s["q"].float().view(B, Hk, G, d)
        at, n = torch.arange(L, device=q.device), s["lens"].long()[:, None]
        seen, away = (at < n)[:, None, None], (n - 1 - at).abs().float()[:, None, None]
    else:
        Lq, Lk = s["max_q"], s["max_k"]
        (q, there), (k, kept), (v, _) = _padded(s["q"], s["q_off"], Lq), _padded(s["k"], s["k_off"], Lk), _padded(s["v"], s["k_off"], Lk)
        nq, nk = (o[1:] - o[:-1] for o in (s["q_off"], s["k_off"]))
        at = torch.arange(Lq, device=q.device) + (nk - nq)[:, None]      # a query's place among the keys
        j = torch.arange(Lk, device=q.device)
        seen = (kept[:, None, :] & there[:, :, None])
        if c["causal"]:
            before = j <= at[:, :, None]
            seen = seen & (before if s["prefix"] is None else before | (j < s["prefix"][:, None, None]))
        seen, away = seen[:, None, None], (at[:, :, None] - j).abs().float()[:, None, None]
        q = q.view(B, Hk, G, Lq, d)
    slope = None if s["slopes"] is None else s["slopes"].view(Hk, G, 1) if c["op"] == "cache" else s["slopes"].view(Hk, G, 1, 1)
    rows = q.reshape(B, Hk, -1, d)
    sc = torch.matmul(rows, k.transpose(2, 3).contiguous()).view(*q.shape[:-1], -1) * scale
    if c["cap"]:
        bent = torch.tanh(sc / c["cap"])
        sc = c["cap"] * bent
    if slope is not None:
        sc = sc - slope * away
    p = _softmax(sc, seen)
    del sc
    flat = p.view(B, Hk, -1, p.shape[-1])
    out = torch.matmul(flat, v)
    if c["op"] == "cache":
        return {"out": out.view(B, Hq, d).to(dt)}
    back = lambda x, here: x.view(B, -1, here.shape[1], d).transpose(1, 2)[here].to(dt)
    if c["op"] == "attn":
        return {"out": back(out, there)}
    do = _padded(s["dout"], s["q_off"], Lq)[0].view(B, Hk, -1, d)
    dv = torch.matmul(flat.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = flat * (dp - (flat * dp).sum(-1, keepdim=True)) * scale
    del dp, p
    if c["cap"]:
        ds = ds * (1 - bent.view(ds.shape).square())
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), rows)
    return {"out": back(out, there), "dq": back(dq, there), "dk": back(dk, kept), "dv": back(dv, kept)}


# ---------------------------------------------------------------------------------------------- in 64 bits
def _exact_rows(x, w, turn):
    """The norm of the last axis and a complex turn of its pairs; turn: [T, pairs], x: [T, H, d] in 64 bits."""
    if w is not None:
        x = x * w / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    return x if turn is None else turn(x)


def exact(c, seed):
    f = torch.float64
    s = prepare(c, seed)
    Hq, Hk, d, G = c["Hq"], c["Hk"], c["d"], c["Hq"] // c["Hk"]
    if c["op"] in ("append", "rope_train"):
        unit = torch.polar(torch.ones((), dtype=f, device=DEV), torch.outer(s["positions"].to(f), s["inv_freq"].to(f)))[:, None]
        n = c["rot"] // 2
        pairs = [(i, i + n) if c["layout"] == "half" else (2 * i, 2 * i + 1) for i in range(n)]
        first, second = (torch.tensor(x, device=DEV) for x in zip(*pairs))

        def turn(x):
            z = torch.complex(x[..., first], x[..., second]) * unit
            return x.index_copy(-1, first, z.real).index_copy(-1, second, z.imag)

        w = [None if s[n] is None else s[n].to(f) for n in ("wq", "wk")]
        if c["op"] == "append":
            q, k = (_exact_rows(s[n].to(f), y, turn) for n, y in zip("qk", w))
            K, V = s["cache_k"].to(f), s["cache_v"].to(f)
            p, seq = s["positions"].cpu().numpy(), s["seqs"].cpu().numpy()
            page = torch.from_numpy(s["table"].cpu().numpy()[seq, p // c["page"]].astype(np.int64)).to(DEV)
            at = torch.from_numpy((p % c["page"]).astype(np.int64)).to(DEV)
            K[page, :, at], V[page, :, at] = k, s["v"].to(f)
            return {"q": q, "cache_k": K, "cache_v": V}
        got = {}
        for n, y in zip("qk", w):  # gradients by differentiation of the formula
            x = s[n].to(f).clone().requires_grad_()
            y = None if y is None else y.clone().requires_grad_()
            o = _exact_rows(x, y, turn)
            o.backward(s["d%s_out" % n].to(f))
            got[n], got["d" + n] = o.detach(), x.grad
            if y is not None:
                got.setdefault("dw", []).append(y.grad)
        if "dw" in got:
            got["dw"] = torch.stack(got["dw"])
        return got
    scale = d ** -0.5
    slopes = torch.zeros(Hq, dtype=f, device=DEV) if s["slopes"] is None else s["slopes"].to(f)

    def weights(q, k, at, h, prefix, causal):
        """(softmax, derivative of the score by the product) of one head's queries [n, d] at places `at` over keys [m, d]."""
        x, j = q @ k.T * scale, torch.arange(k.shape[0], device=DEV)
        slope = torch.full_like(x, scale)
        if c["cap"]:
            t = torch.tanh(x / c["cap"])
            x, slope = t * c["cap"], slope * (1 - t * t)
        x = x - slopes[h] * (at[:, None] - j).abs()
        if causal:
            x[(j > at[:, None]) & (j >= prefix)] = -math.inf
        return torch.nan_to_num(torch.softmax(x, -1), nan=0.0), slope

    if c["op"] == "cache":
        out = torch.zeros(c["B"], Hq, d, dtype=f, device=DEV)
        for b, n in enumerate(s["lens"].tolist()):
            pages = s["table"][b].long()[:(n + c["page"] - 1) // c["page"]]
            K, V = (s[x][pages].to(f).permute(1, 0, 2, 3).reshape(Hk, -1, d)[:, :n] for x in ("cache_k", "cache_v"))
            for h in range(Hq if n else 0):
                p, _ = weights(s["q"][b, h:h + 1].to(f), K[h // G], torch.tensor([n - 1], device=DEV), h, 0, False)
                out[b, h] = p[0] @ V[h // G]
        return {"out": out}
    if c["B"] * Hq > 9000:
        return None
    T, Tk, train = s["q"].shape[0], s["k"].shape[0], c["op"] == "attn_train"
    out, dq = (torch.zeros(T, Hq, d, dtype=f, device=DEV) for _ in range(2))
    dk, dv = (torch.zeros(Tk, Hk, d, dtype=f, device=DEV) for _ in range(2))
    qo, ko = s["q_off"].tolist(), s["k_off"].tolist()
    before = [0] * c["B"] if s["prefix"] is None else s["prefix"].tolist()
    for b in range(c["B"]):
        I, J = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        nq, nk = I.stop - I.start, J.stop - J.start
        if not nq or not nk:
            continue
        at = torch.arange(nq, device=DEV) + nk - nq
        for h in range(Hq):
            q, k, v = s["q"][I, h].to(f), s["k"][J, h // G].to(f), s["v"][J, h // G].to(f)
            p, slope = weights(q, k, at, h, before[b], c["causal"])
            out[I, h] = p @ v
            if train:
                do = s["dout"][I, h].to(f)
                dv[J, h // G] += p.T @ do
                e = p * (do @ v.T - (do * out[I, h]).sum(-1, keepdim=True)) * slope
                dq[I, h] = e @ k
                dk[J, h // G] += e.T @ q
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if train else {"out": out}
