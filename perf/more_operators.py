"""Performance cases of attention with a learned relative position bias (dlrm_seq_attn_bias_*, and dlrm_cache_attn_bias for one new item over
the paged cache), and of attention of several new items of a user over the cache and one another (dlrm_cache_tree_attn).

A case's "op" is what one pass does:
  bias       : attention forward over ragged sequences, scores with a bias by buckets of the distance (scoring)
  bias_train : its forward and backward, the gradient of the bias's table among the outputs
  cache_bias : one new query for each user over the paged cache, with the bias
  tree       : several new items for each user over the paged cache and over one another: a tree in depth-first order, a chain, or
               candidates that see themselves alone ("flat")
The bucket of a distance (a query's place less a key's) is the number of bounds that are at most that distance.
Lengths of the sequences of a case are spread evenly over [lo, hi] and shuffled by the seed, so the work of a case is
the same for every seed.  Sizes are those of workloads/gen.py and of the tests (batches 64, 128, 500, 2048; histories up
to 200 items; widths 16 to 128) and generic ones for long histories."""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _bias(name, op, B, q, k, Hq, Hk, d, dtype, n, far, causal=True, prefix=False, slopes=False, cap=0.0):
    """q, k: (lo, hi) lengths; k None: every item attends over its own sequence.  n buckets, the last from distance `far` on; where
    keys behind the query can be seen (not causal, or a prefix) half of them are for negative distances."""
    c = dict(name=name, op=op, B=B, lo=q[0], hi=q[1], self=k is None, klo=(k or q)[0], khi=(k or q)[1], Hq=Hq, Hk=Hk, d=d,
             dtype=dtype, n=n, far=far, both=prefix or not causal, causal=causal, prefix=prefix, slopes=slopes, cap=cap)
    if not name:
        del c["name"]
    return c


def _cache(name, op, B, lo, hi, items, shape, Hq, Hk, d, dtype, page, n=0, far=0, slopes=False, cap=0.0):
    """lo, hi: items in the cache; items: (lo, hi) new ones; n: buckets of the bias, 0 for none."""
    c = dict(name=name, op=op, B=B, lo=lo, hi=hi, ilo=items[0], ihi=items[1], shape=shape, Hq=Hq, Hk=Hk, d=d, dtype=dtype, page=page,
             n=n, far=far, both=False, slopes=slopes, cap=cap)
    if not name:
        del c["name"]
    return c


def listed():
    one = (1, 1)
    return [
        # the smallest training batch: 128 users with next to no history, some with none
        _bias("bias_train_tiny", "bias_train", 128, (0, 20), None, 2, 2, 16, "f32", 8, 16),
        # ordinary histories in bf16
        _bias("bias_train_history", "bias_train", 2048, (1, 200), None, 4, 4, 64, "bf16", 32, 128),
        # long histories, capped scores, four query heads to a key head, buckets that widen over the whole length: the largest
        _bias("bias_train_long", "bias_train", 8, (2048, 4096), None, 16, 4, 128, "bf16", 64, 2048, cap=30.0),
        # odd sizes in fp32, the first quarter of a history (profile items) seen by all of it: distances of both signs
        _bias("bias_train_odd_f32", "bias_train", 13, (1, 1999), None, 6, 3, 72, "f32", 33, 300, prefix=True),
        # candidates scored against histories, some of them empty; two key heads, an odd width
        _bias("bias_candidates_f16", "bias", 500, (1, 40), (0, 1000), 8, 2, 40, "f16", 32, 128, causal=False),
        # 64 users with short histories in fp32, one new item each: latency
        _cache("cache_bias_serve_f32", "cache_bias", 64, 1, 200, one, "chain", 4, 4, 64, "f32", 16, n=32, far=128),
        # a full serving batch of mixed lengths, one new item each
        _cache("cache_bias_mixed", "cache_bias", 256, 1, 8192, one, "chain", 16, 4, 128, "bf16", 32, n=64, far=2048, cap=50.0),
        # eight drafted items for each of 64 users with short histories: latency
        _cache("tree_serve_b64", "tree", 64, 1, 200, (8, 8), "tree", 8, 2, 64, "bf16", 64),
        # candidates of 500 users, each seen by itself alone, over histories of which some are empty
        _cache("tree_candidates_f16", "tree", 500, 0, 1000, (1, 40), "flat", 8, 2, 40, "f16", 16, slopes=True),
        # one user with a very long history and a tree of 64 drafts: the length is all there is to split
        _cache("tree_one_long", "tree", 1, 131072, 131072, (64, 64), "tree", 16, 4, 128, "bf16", 64),
        # a piece of each of 13 long prompts after the pieces before it, fp32, an odd width
        _cache("tree_prompt_f32", "tree", 13, 1, 1999, (1, 129), "chain", 6, 3, 72, "f32", 8, n=16, far=100),
        # a full batch of mixed lengths with trees of up to 60 drafts, learned bias, capped: the largest of its kind
        _cache("tree_batch_mixed", "tree", 128, 1, 8192, (1, 60), "tree", 16, 4, 128, "bf16", 32, n=64, far=2048, cap=50.0),
    ]


def draw(rng):
    """Another case of the same ranges: any operator, batch, lengths, heads, width, type and mask, at most as much work as
    the largest listed case of its kind."""
    logu = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    while True:
        op = rng.choice(["bias", "bias_train", "bias_train", "cache_bias", "tree", "tree"])
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        Hk = rng.choice([1, 2, 3, 4, 8])
        Hq = Hk * rng.choice([1, 1, 2, 4, 5, 8])
        d = 8 * logu(1, 16)
        B = logu(1, 2048)
        n, far = logu(2, 128), logu(128, 8192)
        slopes, cap = rng.random() < 0.2, rng.choice([0.0, 0.0, 30.0])
        if op in ("bias", "bias_train"):
            least = 1 if op == "bias" else 2  # (a row that sees one key alone has no gradient but rounding)
            hi = logu(least, 4096)
            alone = rng.random() < 0.7
            khi = hi if alone else logu(least, 4096)
            causal = rng.random() < 0.7
            c = _bias("", op, B, (rng.choice([0, 1, hi // 2, hi]), hi), None if alone else (rng.choice([0, 1, khi]), khi), Hq, Hk, d, dtype, n, far,
                      causal=causal, prefix=causal and rng.random() < 0.3, slopes=slopes, cap=cap)
            if B * Hq * hi * khi <= 8 * 16 * 4096 * 4096 and B * (hi + khi) * Hq * d <= 2048 * 400 * 16 * 128 and B * (hi + khi) <= 2048 * 800:
                return c
            continue
        hi, top = logu(1, 131072), 1 if op == "cache_bias" else logu(1, 256)
        with_bias = op == "cache_bias" or rng.random() < 0.5
        c = _cache("", op, B, rng.choice([0, 1, hi // 2, hi]), hi, (rng.choice([1, max(1, top // 2), top]), top), rng.choice(["tree", "tree", "chain", "flat"]),
                   Hq, Hk, d, dtype, 2 ** rng.randint(3, 7), n=n if with_bias else 0, far=far if with_bias else 0, slopes=slopes, cap=cap)
        if B * hi * Hk * d <= 128 * 8192 * 4 * 128 and B * (hi + top) * Hq * top <= 128 * 8192 * 16 * 60 and B * top * Hq * d <= 128 * 60 * 16 * 128:
            return c


# ---------------------------------------------------------------------------------------------- sizes
def _even(n, lo, hi):
    return np.rint(np.linspace(hi, lo, n)).astype(np.int64)


def _lengths(c):
    return _even(c["B"], c["lo"], c["hi"])


def _new(c):
    """New items of each sequence, in an order of their own beside the lengths of the caches."""
    return np.random.RandomState(7).permutation(_even(c["B"], c["ilo"], c["ihi"]))


def _cols(c):
    return max(1, (c["hi"] + c["page"] - 1) // c["page"])


def _bounds(c):
    """n - 1 ascending bounds: the distances from 1 on one by one for half of the buckets, then by equal factors up to `far`.  For both signs
    as many again: a distance of -x is in a bucket of its own where x is."""
    def up(m):  # m bounds
        e = (m + 1) // 2
        b = list(range(1, e + 1))
        for k in range(1, m - e + 1):
            b.append(max(b[-1] + 1, int(math.ceil(e * (max(c["far"], e + 1) / e) ** (k / (m - e))))))
        return b
    m = c["n"] - 1
    return [1 - x for x in reversed(up(m // 2))] + up(m - m // 2) if c["both"] else up(m)


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
    lens = _lengths(c)
    T = int(lens.sum())
    if c["op"] == "cache_bias":
        return {"bytes": T * Hk * d * e * 2 + 2 * c["B"] * Hq * d * e, "flops": T * Hq * d * 4}
    if c["op"] == "tree":
        new = _new(c)
        N = int(new.sum())  # (pairs of new items are counted as if each saw half of the others)
        return {"bytes": T * Hk * d * e * 2 + 2 * N * (Hq + Hk) * d * e, "flops": float((new * (lens + new / 2)).sum()) * Hq * d * 4}
    Tk = int(_even(c["B"], c["klo"], c["khi"]).sum())
    rows = T * Hq * d * e * 2 + Tk * Hk * d * e * 2
    if c["op"] == "bias":
        return {"bytes": rows, "flops": _pairs(c) * Hq * d * 4}
    return {"bytes": 2 * rows + T * Hq * d * e * 2 + 2 * Hq * c["n"] * 4, "flops": _pairs(c) * Hq * d * 14}


# ---------------------------------------------------------------------------------------------- inputs
def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=DEV)


def _tree(rng, n, shape):
    """(last, depth) of n items in depth-first order: the last item that sees item j, and how far j is from the cache."""
    if shape == "flat":
        return list(range(n)), [0] * n
    if shape == "chain":
        return [n - 1] * n, list(range(n))
    last, depth, path = [0] * n, [0] * n, []
    for i, r in enumerate(rng.random_sample(n)):
        keep = int((len(path) + 1) * (1 - r * r))  # mostly the newest item or one near it is drafted on
        for j in path[keep:]:
            last[j] = i - 1
        del path[keep:]
        depth[i] = len(path)
        path.append(i)
    for j in path:
        last[j] = n - 1
    return last, depth


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 32))
    dt, B, Hq, Hk, d = DTYPES[c["dtype"]], c["B"], c["Hq"], c["Hk"], c["d"]
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dt)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=t)
    s = {"c": c}
    order = rng.permutation(B)
    lens = _lengths(c)[order]
    s["table"] = s["bounds"] = None
    if c["n"]:
        s["table"] = torch.randn(Hq, c["n"], generator=g, device=DEV)
        s["bounds"] = dev(np.array(_bounds(c), dtype=np.int32), torch.int32)
    s["slopes"] = _slopes(Hq) if c["slopes"] else None
    if c["op"] in ("cache_bias", "tree"):
        cols = _cols(c)
        # the pages of B users, in the order in which a pool that has been in use for a while hands them out
        s["pages"] = torch.randperm(B * cols, generator=g, device=DEV).to(torch.int32).view(B, cols)
        s["cache_k"], s["cache_v"] = rand(B * cols, Hk, c["page"], d), rand(B * cols, Hk, c["page"], d)
        s["lens"] = dev(lens, torch.int32)
        if c["op"] == "cache_bias":
            s["q"], s["out"] = rand(B, Hq, d), torch.empty(B, Hq, d, dtype=dt, device=DEV)
        else:
            new = _new(c)[order]
            T = int(new.sum())
            shapes = [_tree(rng, int(n), c["shape"]) for n in new]
            qkv = rand(T, Hq + 2 * Hk, d)
            s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
            s["out"] = torch.empty(T, Hq, d, dtype=dt, device=DEV)
            s["off"], s["max_items"] = dev(_offsets(new), torch.int64), int(new.max())
            s["last"] = dev(np.concatenate([t[0] for t in shapes]), torch.int32)
            s["positions"] = dev(np.concatenate([t[1] for t in shapes]) + np.repeat(lens, new), torch.int32)
    else:
        T = int(lens.sum())
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
        s["out"], s["lse"] = torch.empty(T, Hq, d, dtype=dt, device=DEV), torch.empty(Hq, T, device=DEV)
        s["max_q"], s["max_k"] = int(lens.max()), int(klens.max())
        if c["op"] == "bias_train":
            s["dout"], s["dq"] = rand(T, Hq, d), torch.empty(T, Hq, d, dtype=dt, device=DEV)
            s["dk"], s["dv"] = (torch.empty(Tk, Hk, d, dtype=dt, device=DEV) for _ in range(2))
            s["dtable"] = torch.empty_like(s["table"])
    if own:
        import paper_1906_00091_amd as hot
        s["bias"] = hot.RelBias(s["table"], s["bounds"]) if c["n"] else None
        if c["op"] in ("cache_bias", "tree"):
            s["cache"], s["top"] = hot.KvCache(s["cache_k"], s["cache_v"], s["pages"]), max(1, c["hi"])
            if c["op"] == "cache_bias":
                s["ws"] = hot.alloc_cache_attn_bias_workspace(s["cache"], Hq, s["top"])
            else:
                s["items"] = hot.NewItems(s["off"], T, s["max_items"], last=s["last"], positions=s["positions"])
                s["ws"] = hot.alloc_cache_tree_attn_workspace(s["cache"], Hq, s["top"], s["items"])
        else:
            s["plan"] = hot.SeqBatch(s["q_off"], s["k_off"], T, Tk, s["max_q"], s["max_k"], causal=c["causal"], prefix=s["prefix"],
                                     slopes=s["slopes"], cap=c["cap"])
            if c["op"] == "bias_train":
                s["ws"] = hot.alloc_seq_attn_bias_workspace(s["plan"], s["bias"], Hq, Hk, d)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)(s, s["c"])


def _own(s, c):
    import paper_1906_00091_amd as hot
    if c["op"] == "cache_bias":
        hot.dlrm_cache_attn_bias(s["cache"], s["lens"], s["top"], s["bias"], s["q"], s["out"], s["ws"], slopes=s["slopes"], cap=c["cap"])
        return {"out": s["out"]}
    if c["op"] == "tree":
        hot.dlrm_cache_tree_attn(s["cache"], s["lens"], s["top"], s["items"], s["q"], s["k"], s["v"], s["out"], s["ws"], bias=s["bias"],
                                 slopes=s["slopes"], cap=c["cap"])
        return {"out": s["out"]}
    hot.dlrm_seq_attn_bias_fwd(s["plan"], s["bias"], s["q"], s["k"], s["v"], s["out"], s["lse"])
    if c["op"] == "bias":
        return {"out": s["out"]}
    hot.dlrm_seq_attn_bias_bwd(s["plan"], s["bias"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], s["dtable"],
                               s["ws"])
    return {"out": s["out"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dtable": s["dtable"]}


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


def _buckets(s, away):
    return torch.bucketize(away, s["bounds"].long(), right=True)


def _scored(s, c, sc, away):
    """Scores [B, Hk, G, queries, keys] from the products, and tanh of the capped ones; away: distances [B, queries, keys]."""
    bent, (B, Hk, G, *_) = None, sc.shape
    sc = sc * c["d"] ** -0.5
    if c["cap"]:
        bent = torch.tanh(sc / c["cap"])
        sc = c["cap"] * bent
    if s["slopes"] is not None:
        sc = sc - s["slopes"].view(Hk, G, 1, 1) * away.abs().float()[:, None, None]
    if s["table"] is not None:
        sc += s["table"][:, _buckets(s, away)].transpose(0, 1).reshape(sc.shape)
    return sc, bent


def _plain(s, c):
    dt, Hq, Hk, d, B = DTYPES[c["dtype"]], c["Hq"], c["Hk"], c["d"], c["B"]
    G = Hq // Hk
    product = lambda a, b: torch.matmul(a, b.transpose(2, 3).contiguous())
    if c["op"] in ("cache_bias", "tree"):
        L = s["pages"].shape[1] * c["page"]
        k, v = (s[n][s["pages"].long()].float().transpose(1, 2).reshape(B, Hk, L, d) for n in ("cache_k", "cache_v"))
        n, at = s["lens"].long()[:, None], torch.arange(L, device=k.device)
        cached = (at < n)[:, None]
        if c["op"] == "cache_bias":
            q = s["q"].float().view(B, Hk, G, d)
            sc, _ = _scored(s, c, product(q, k).view(B, Hk, G, 1, L), (n - 1 - at)[:, None])
            out = torch.matmul(_softmax(sc, cached[:, None, None]).view(B, Hk, G, L), v)
            return {"out": out.view(B, Hq, d).to(dt)}
        N = s["max_items"]
        (q, there), (nk, _), (nv, _) = (_padded(s[x], s["off"], N) for x in "qkv")
        rows = (s["off"][:-1, None] + torch.arange(N, device=k.device)).clamp(max=s["q"].shape[0] - 1)
        pos, last, i = s["positions"].long()[rows], s["last"].long()[rows], torch.arange(N, device=k.device)
        old = there[:, :, None] & cached
        new = there[:, :, None] & there[:, None] & (i <= i[:, None]) & (i[:, None] <= last[:, None])
        q = q.reshape(B, Hk, G * N, d)
        sc = torch.cat([product(q, k), product(q, nk)], -1).view(B, Hk, G, N, L + N)
        away = torch.cat([pos[:, :, None] - at, pos[:, :, None] - pos[:, None]], -1)
        sc, _ = _scored(s, c, sc, away)
        p = _softmax(sc, torch.cat([old, new], -1)[:, None, None]).view(B, Hk, G * N, L + N)
        out = torch.matmul(p[..., :L], v) + torch.matmul(p[..., L:], nv)
        return {"out": out.view(B, Hq, N, d).transpose(1, 2)[there].to(dt)}

    Lq, Lk = s["max_q"], s["max_k"]
    (q, there), (k, kept), (v, _) = _padded(s["q"], s["q_off"], Lq), _padded(s["k"], s["k_off"], Lk), _padded(s["v"], s["k_off"], Lk)
    nq, nk = (o[1:] - o[:-1] for o in (s["q_off"], s["k_off"]))
    at = torch.arange(Lq, device=q.device) + (nk - nq)[:, None]      # a query's place among the keys
    j = torch.arange(Lk, device=q.device)
    seen = (kept[:, None, :] & there[:, :, None])
    if c["causal"]:
        before = j <= at[:, :, None]
        seen = seen & (before if s["prefix"] is None else before | (j < s["prefix"][:, None, None]))
    rows = q.reshape(B, Hk, G * Lq, d)
    sc, bent = _scored(s, c, product(rows, k).view(B, Hk, G, Lq, Lk), at[:, :, None] - j)
    flat = _softmax(sc, seen[:, None, None]).view(B, Hk, G * Lq, Lk)
    del sc
    out = torch.matmul(flat, v)
    back = lambda x, here: x.reshape(B, -1, here.shape[1], d).transpose(1, 2)[here].to(dt)
    if c["op"] == "bias":
        return {"out": back(out, there)}
    do = _padded(s["dout"], s["q_off"], Lq)[0].reshape(B, Hk, G * Lq, d)
    dv = torch.matmul(flat.transpose(2, 3).contiguous(), do)
    dp = product(do, v)
    ds = flat * (dp - (flat * dp).sum(-1, keepdim=True))
    del dp, flat
    dtable = _by_bucket(s, ds.view(B, Hq, Lq, Lk), nk - nq)
    ds *= d ** -0.5
    if c["cap"]:
        ds = ds * (1 - bent.view(ds.shape).square())
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), rows)
    return {"out": back(out, there), "dq": back(dq, there), "dk": back(dk, kept), "dv": back(dv, kept), "dtable": dtable}


def _by_bucket(s, x, shift):
    """Sums of x [B, H, Lq, Lk] over pairs whose distance i + shift - j is in a bucket, [H, n]: first along the diagonals (a row written one
    element further to the right than the row before it turns them into columns), then by the diagonals' buckets in 64 bits."""
    B, H, Lq, Lk = x.shape
    W = Lq + Lk - 1
    x = torch.nn.functional.pad(x.flip(-1), (0, Lq)).flatten(2)[..., :Lq * W].view(B, H, Lq, W).sum(2)
    away = torch.arange(W, device=x.device) - (Lk - 1) + shift[:, None]
    which = _buckets(s, away)[..., None] == torch.arange(s["table"].shape[1], device=x.device)
    return torch.matmul(x.double(), which.double()).sum(0).float()


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(c, seed):
    f = torch.float64
    s = prepare(c, seed)
    Hq, Hk, d, G = c["Hq"], c["Hk"], c["d"], c["Hq"] // c["Hk"]
    bounds = None if s["bounds"] is None else s["bounds"].long()
    inf = torch.full((1,), 1 << 40, dtype=torch.int64, device=DEV)
    edges = None if bounds is None else torch.cat([-inf, bounds, inf])

    def weights(q, k, away, h, seen):
        """(softmax, derivative of the score by the product) of one head's queries [n, d] at distances `away` [n, m] from keys [m, d]."""
        x = q @ k.T * d ** -0.5
        slope = torch.full_like(x, d ** -0.5)
        if c["cap"]:
            t = torch.tanh(x / c["cap"])
            x, slope = t * c["cap"], slope * (1 - t * t)
        if s["slopes"] is not None:
            x = x - s["slopes"][h].to(f) * away.abs()
        if bounds is not None:
            x = x + s["table"][h].to(f)[torch.searchsorted(bounds, away.contiguous(), right=True)]
        x = x.masked_fill(~seen, -math.inf)
        return torch.nan_to_num(torch.softmax(x, -1), nan=0.0), slope

    if c["op"] in ("cache_bias", "tree"):
        if c["B"] * Hq > 9000:
            return None
        out = torch.zeros(s["q"].shape, dtype=f, device=DEV)
        off = list(range(c["B"] + 1)) if c["op"] == "cache_bias" else s["off"].tolist()
        for b, n in enumerate(s["lens"].tolist()):
            I = slice(off[b], off[b + 1])
            m = I.stop - I.start
            pages = s["pages"][b].long()[:(n + c["page"] - 1) // c["page"]]
            K, V = (s[x][pages].to(f).permute(1, 0, 2, 3).reshape(Hk, -1, d)[:, :n] for x in ("cache_k", "cache_v"))
            if c["op"] == "cache_bias":
                pos, place = torch.tensor([n - 1], device=DEV), torch.arange(n, device=DEV)
                seen = torch.ones(1, n, dtype=torch.bool, device=DEV)
            else:
                K, V = (torch.cat([x, s[y][I].to(f).transpose(0, 1)], 1) for x, y in ((K, "k"), (V, "v")))
                pos, i = s["positions"][I].long(), torch.arange(m, device=DEV)
                place = torch.cat([torch.arange(n, device=DEV), pos])
                seen = torch.cat([torch.ones(m, n, dtype=torch.bool, device=DEV), (i[:, None] >= i) & (i[:, None] <= s["last"][I].long())], 1)
            for h in range(Hq if seen.numel() else 0):
                p, _ = weights(s["q"][I, h].to(f), K[h // G], pos[:, None] - place, h, seen)
                out[I, h] = p @ V[h // G]
        return {"out": out}
    if c["B"] * Hq > 9000:
        return None
    T, Tk, train = s["q"].shape[0], s["k"].shape[0], c["op"] == "bias_train"
    out, dq = (torch.zeros(T, Hq, d, dtype=f, device=DEV) for _ in range(2))
    dk, dv = (torch.zeros(Tk, Hk, d, dtype=f, device=DEV) for _ in range(2))
    dtable = torch.zeros(Hq, c["n"], dtype=f, device=DEV)
    qo, ko = s["q_off"].tolist(), s["k_off"].tolist()
    before = [0] * c["B"] if s["prefix"] is None else s["prefix"].tolist()
    for b in range(c["B"]):
        I, J = slice(qo[b], qo[b + 1]), slice(ko[b], ko[b + 1])
        nq, nk = I.stop - I.start, J.stop - J.start
        if not nq or not nk:
            continue
        at, j = torch.arange(nq, device=DEV) + nk - nq, torch.arange(nk, device=DEV)
        away = at[:, None] - j
        seen = (away >= 0) | (j < before[b]) if c["causal"] else torch.ones_like(away, dtype=torch.bool)
        # keys whose distance is at least an edge come before this one
        ends = (at[:, None] - edges + 1).clamp(0, nk)
        for h in range(Hq):
            q, k, v = s["q"][I, h].to(f), s["k"][J, h // G].to(f), s["v"][J, h // G].to(f)
            p, slope = weights(q, k, away, h, seen)
            out[I, h] = p @ v
            if train:
                do = s["dout"][I, h].to(f)
                dv[J, h // G] += p.T @ do
                e = p * (do @ v.T - (do * out[I, h]).sum(-1, keepdim=True))
                upto = torch.cat([torch.zeros(nq, 1, dtype=f, device=DEV), e.cumsum(1)], 1).gather(1, ends).sum(0)
                dtable[h] += upto[:-1] - upto[1:]
                e = e * slope
                dq[I, h] = e @ k
                dk[J, h // G] += e.T @ q
    return {"out": out, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable} if train else {"out": out}
