"""Operators that read a history in order (dlrm_qk_rope_*, dlrm_seq_attn_*, dlrm_cache_attn) against plain 64-bit forms
(history_ref), with elementwise bounds."""
import math
import os
import sys

import numpy as np
import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def placed(x, layout):
    """x [T, H, d] on the device, in one of the layouts that a caller may have; what lies between the rows is NaN."""
    T, H, d = x.shape
    if layout == "rows":
        return x.to(DEV)
    if layout == "packed":      # heads side by side with others in a wider row
        b = torch.full((T, H + 3, d), NAN, dtype=x.dtype, device=DEV)
        v = b[:, 1:1 + H]
    elif layout == "heads":     # head by head
        b = torch.full((H, T, d), NAN, dtype=x.dtype, device=DEV)
        v = b.transpose(0, 1)
    else:                       # "wide": rows wider than d
        b = torch.full((T, H, d + 8), NAN, dtype=x.dtype, device=DEV)
        v = b[..., :d]
    v.copy_(x)
    return v


# ------------------------------------------------------------------------------------------------ norm and rotation
ROPE = [
    # dtype, T, Hq, Hk, d, rot, layout, norm, positions up to, where the rows lie
    ("f32", 1, 1, 1, 8, 8, "half", True, 5, "rows"),
    ("f32", 37, 4, 2, 64, 64, "interleaved", True, 100, "packed"),
    ("f32", 129, 3, 1, 72, 20, "half", True, 1 << 20, "heads"),      # partners in other chunks' middles
    ("f32", 50, 2, 2, 128, 0, "half", True, 9, "wide"),              # norm alone
    ("f16", 65, 8, 8, 64, 32, "interleaved", False, 2000, "packed"),  # rotation alone
    ("f16", 33, 5, 1, 40, 38, "half", True, 300, "rows"),
    ("bf16", 64, 8, 2, 64, 64, "half", True, 2000, "packed"),
    ("bf16", 700, 16, 4, 128, 128, "half", True, 1 << 24, "packed"),
    ("bf16", 3, 2, 1, 24, 2, "interleaved", True, 2147483647, "heads"),
    ("bf16", 17, 7, 7, 104, 90, "half", False, 64, "wide"),
    ("bf16", 9, 3, 0, 128, 64, "half", True, 64, "rows"),            # queries alone
]


def rope_case(i):
    dt, T, Hq, Hk, d, rot, layout, norm, top, where = ROPE[i]
    g = gen(100 + i)
    dt = DT[dt]
    x = {"q": rand(g, T, Hq, d, dtype=dt), "k": rand(g, T, max(Hk, 1), d, dtype=dt)}
    x["q"][0] = 0                                                    # a row of zeros has a norm of eps
    w = {n: 1 + 0.1 * rand(g, d) if norm else None for n in "qk"}
    pos = torch.randint(0, top, (T,), generator=g, dtype=torch.int64).to(torch.int32)
    f = hot.rope_frequencies(rot, stretch=2.0)
    up = lambda t: None if t is None else t.to(DEV)
    plan = hot.QkRope(pos.to(DEV), Hq, Hk, d, inv_freq=f.to(DEV) if rot else None, rot=rot, eps=1e-5, mscale=1.25,
                      layout=hot.ROPE_HALF if layout == "half" else hot.ROPE_INTERLEAVED, wq=up(w["q"]), wk=up(w["k"]))
    return dt, x, w, (pos, f, rot, layout, 1e-5, 1.25), plan, where, Hk


def rope_bound(dt, x, w, y, mscale, d):
    """One rounding of y, and fp32: the norm's sum of d squares, sine and cosine to 2^-22, two products."""
    n = x.double().abs() if w is None else (x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-5) * w.double()).abs()
    return ref.UNIT[dt] * y.abs() + (d + 24) * ref.E32 * mscale * 2 * n.amax(-1, keepdim=True) + ref.TINY[dt]


@pytest.mark.parametrize("i", range(len(ROPE)))
def test_norm_and_rotation_forward(i):
    dt, x, w, how, plan, where, Hk = rope_case(i)
    d = x["q"].shape[2]
    q, k = placed(x["q"], where), placed(x["k"], where)
    qo, ko = placed(torch.zeros_like(x["q"]), where), placed(torch.zeros_like(x["k"]), where)
    hot.dlrm_qk_rope_fwd(plan, q, k if Hk else None, qo, ko if Hk else None)
    for n, got in (("q", qo), ("k", ko)) if Hk else (("q", qo),):
        y = ref.rope(x[n], w[n], *how)
        ref.close(got, y, rope_bound(dt, x[n], w[n], y, how[5], d), n)
    hot.dlrm_qk_rope_fwd(plan, q, k if Hk else None, q, k if Hk else None)   # in place: the same bits
    assert torch.equal(q, qo) and (not Hk or torch.equal(k, ko))


@pytest.mark.parametrize("i", range(len(ROPE)))
def test_norm_and_rotation_backward(i):
    dt, x, w, how, plan, where, Hk = rope_case(i)
    g = gen(500 + i)
    d, T = x["q"].shape[2], x["q"].shape[0]
    dy = {n: rand(g, *x[n].shape, dtype=dt) for n in "qk"}
    dev = {n: placed(x[n], where) for n in "qk"}
    ddev = {n: placed(dy[n], where) for n in "qk"}
    out = {n: placed(torch.zeros_like(x[n]), where) for n in "qk"}
    dw = torch.full((2, d), NAN, device=DEV)
    ws = hot.alloc_qk_rope_workspace(plan)
    keys = lambda t: t["k"] if Hk else None

    def call(to):
        hot.dlrm_qk_rope_bwd(plan, dev["q"], keys(dev), ddev["q"], keys(ddev), to["q"], keys(to), dw[0] if w["q"] is not None else None,
                             dw[1] if w["k"] is not None else None, ws)
    call(out)
    first = dw.clone()
    for j, n in enumerate("qk" if Hk else "q"):
        dx, dwn = ref.rope_grad(x[n], w[n], dy[n], *how)
        r = torch.ones(1) if w[n] is None else 1 / torch.sqrt(x[n].double().square().mean(-1, keepdim=True) + how[4])
        gmag = how[5] * 2 * dy[n].double().abs().amax(-1, keepdim=True) * (1 if w[n] is None else w[n].double().abs().amax())
        size = r.double() * gmag * (1 + (x[n].double() * r).abs().amax(-1, keepdim=True))
        ref.close(out[n], dx, ref.UNIT[dt] * dx.abs() + 2 * (d + 24) * ref.E32 * size + ref.TINY[dt], "d" + n)
        if dwn is not None:
            xn = (x[n].double() * r).abs()
            terms = (gmag * xn).sum((0, 1))       # |terms| of the sum; roundings along any path through the joining tree
            ref.close(dw[j], dwn, (d + 24 + T * x[n].shape[1]) * ref.E32 * terms + 1e-30, "dw" + n)
    call(ddev)                                    # in place of the upstream gradients; bit for bit
    assert torch.equal(ddev["q"], out["q"]) and (not Hk or torch.equal(ddev["k"], out["k"]))
    rows = [j for j, n in enumerate("qk" if Hk else "q") if w[n] is not None]
    assert torch.equal(dw[rows], first[rows])


@pytest.mark.parametrize("dtype,d,Hq,Hk,layout", [("bf16", 8, 20, 4, "interleaved"), ("f16", 16, 3, 5, "half"), ("bf16", 24, 1, 1, "half"), ("f32", 8, 5, 2, "half")])
def test_many_items_of_narrow_rows(dtype, d, Hq, Hk, layout):
    g, dt, T, rot = gen(d), DT[dtype], 70001, 6
    x = {"q": rand(g, T, Hq, d, dtype=dt), "k": rand(g, T, Hk, d, dtype=dt)}
    dy = {n: rand(g, *x[n].shape, dtype=dt) for n in "qk"}
    w = 1 + 0.1 * rand(g, 2, d)
    pos, f = torch.arange(T, dtype=torch.int32) % 1000, hot.rope_frequencies(rot)
    how = (pos, f, rot, layout, 1e-5, 1.0)
    wd = w.to(DEV)
    plan = hot.QkRope(pos.to(DEV), Hq, Hk, d, inv_freq=f.to(DEV), rot=rot, eps=1e-5, wq=wd[0], wk=wd[1],
                      layout=hot.ROPE_HALF if layout == "half" else hot.ROPE_INTERLEAVED)
    X, DY = ({n: placed(t[n], "packed") for n in "qk"} for t in (x, dy))
    out, dx = ({n: torch.empty(T, x[n].shape[1], d, dtype=dt, device=DEV) for n in "qk"} for _ in range(2))
    dw = torch.empty(2, d, device=DEV)
    hot.dlrm_qk_rope_fwd(plan, X["q"], X["k"], out["q"], out["k"])
    hot.dlrm_qk_rope_bwd(plan, X["q"], X["k"], DY["q"], DY["k"], dx["q"], dx["k"], dw[0], dw[1], hot.alloc_qk_rope_workspace(plan))
    for j, n in enumerate("qk"):
        y = ref.rope(x[n], w[j], *how)
        ref.close(out[n], y, rope_bound(dt, x[n], w[j], y, 1.0, d), n)
        want, dwn = ref.rope_grad(x[n], w[j], dy[n], *how)
        r = 1 / torch.sqrt(x[n].double().square().mean(-1, keepdim=True) + 1e-5)
        xn = (x[n].double() * r).abs()
        gmag = 2 * dy[n].double().abs().amax(-1, keepdim=True) * w[j].double().abs().amax()
        ref.close(dx[n], want, ref.UNIT[dt] * want.abs() + 2 * (d + 24) * ref.E32 * r * gmag * (1 + xn.amax(-1, keepdim=True)) + ref.TINY[dt], "d" + n)
        # sums of a thousand terms a lane, then of the lanes and workgroups: n e32 times the terms is a bound on any of it
        ref.close(dw[j], dwn, (d + 24 + 2000) * ref.E32 * (gmag * xn).sum((0, 1)) + 1e-30, "dw" + n)


def test_no_items_leave_gradients_of_zero():
    plan = hot.QkRope(torch.empty(0, dtype=torch.int32, device=DEV), 2, 2, 16, wq=torch.ones(16, device=DEV), wk=torch.ones(16, device=DEV))
    e = torch.empty(0, 2, 16, device=DEV)
    dw = torch.ones(2, 16, device=DEV)
    hot.dlrm_qk_rope_fwd(plan, e, e, e, e)
    hot.dlrm_qk_rope_bwd(plan, e, e, e, e, e, e, dw[0], dw[1], hot.alloc_qk_rope_workspace(plan))
    assert not dw.any()


# ------------------------------------------------------------------------------------------------ into the cache
@pytest.mark.parametrize("dtype,page,Hk,d,rot,layout", [("f32", 1, 2, 16, 16, "half"), ("bf16", 16, 2, 64, 64, "half"),
                                                       ("f16", 8, 3, 40, 20, "interleaved"), ("bf16", 64, 1, 128, 100, "half")])
def test_append_stores_what_the_forward_gives_and_nothing_else(dtype, page, Hk, d, rot, layout):
    g = gen(7)
    dt, Hq = DT[dtype], 2 * Hk
    start, new = [0, 5, 63, 0, 17], [3, 1, 70, 0, 31]
    B, cols = len(new), (140 + page - 1) // page
    table = torch.randperm(B * cols + 3, generator=g)[:B * cols].view(B, cols).to(torch.int32)
    table[4, 20 // page] = -1                                        # a page that is not there
    T = sum(new) + 2
    seqs = torch.tensor(sum(([s] * n for s, n in enumerate(new)), []) + [-1, B], dtype=torch.int32)   # two items of no sequence
    pos = torch.tensor(sum((list(range(a, a + n)) for a, n in zip(start, new)), []) + [0, 0], dtype=torch.int32)
    q, k, v = (rand(g, T, H, d, dtype=dt) for H in (Hq, Hk, Hk))
    w = 1 + 0.1 * rand(g, 2, d)
    f = hot.rope_frequencies(rot)
    plan = hot.QkRope(pos.to(DEV), Hq, Hk, d, inv_freq=f.to(DEV), layout=hot.ROPE_HALF if layout == "half" else hot.ROPE_INTERLEAVED,
                      wq=w[0].to(DEV).contiguous(), wk=w[1].to(DEV).contiguous())
    qo, ko, qa = (torch.empty(T, H, d, dtype=dt, device=DEV) for H in (Hq, Hk, Hq))
    hot.dlrm_qk_rope_fwd(plan, q.to(DEV), k.to(DEV), qo, ko)
    pool = torch.full((2, B * cols + 3, Hk, page, d), 7.0, dtype=dt, device=DEV)
    want = pool.clone().cpu()
    hot.dlrm_qk_rope_append(plan, placed(q, "packed"), placed(k, "heads"), placed(v, "packed"), qa,
                            hot.KvCache(pool[0], pool[1], table.to(DEV)), seqs.to(DEV))
    assert torch.equal(qa, qo)
    kc = ko.cpu()
    for t in range(T):
        s, p = int(seqs[t]), int(pos[t])
        if 0 <= s < B and int(table[s, p // page]) >= 0:
            want[0, int(table[s, p // page]), :, p % page] = kc[t]
            want[1, int(table[s, p // page]), :, p % page] = v[t]
    assert torch.equal(pool.cpu(), want)


@pytest.mark.parametrize("T,Hq,Hk", [(1, 3, 5), (3000, 2, 7), (9000, 4, 5), (40000, 8, 8)])
def test_append_of_any_number_of_items(T, Hq, Hk):
    """From every head of an item on its own to all heads of an item in one walk (fp32, d 16: four lanes a row)."""
    g, d, page = gen(T), 16, 8
    q, k, v = (rand(g, T, H, d).to(DEV) for H in (Hq, Hk, Hk))
    n = (T + page - 1) // page
    table = torch.randperm(n, generator=g).view(1, n).to(torch.int32)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    plan = hot.QkRope(pos, Hq, Hk, d, inv_freq=hot.rope_frequencies(d, device=DEV))
    qo, ko, qa = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    hot.dlrm_qk_rope_fwd(plan, q, k, qo, ko)
    how = (pos.cpu(), hot.rope_frequencies(d), d, "half", 1e-6, 1.0)
    for a, b in ((q, qo), (k, ko)):
        y = ref.rope(a.cpu(), None, *how)
        ref.close(b, y, rope_bound(torch.float32, a.cpu(), None, y, 1.0, d), "rows")
    pool = torch.full((2, n, Hk, page, d), 7.0, device=DEV)
    hot.dlrm_qk_rope_append(plan, q, k, v, qa, hot.KvCache(pool[0], pool[1], table.to(DEV)), torch.zeros(T, dtype=torch.int32, device=DEV))
    assert torch.equal(qa, qo)
    at = table[0].to(DEV).long()
    for x, y in ((ko, pool[0]), (v, pool[1])):
        rows = y[at].transpose(1, 2).reshape(n * page, Hk, d)
        assert torch.equal(rows[:T], x) and (rows[T:] == 7.0).all()


def test_items_past_the_table_are_not_stored():
    pool = torch.zeros(2, 4, 1, 8, 16, device=DEV)
    x = torch.ones(2, 1, 16, device=DEV)
    plan = hot.QkRope(torch.tensor([16, -1], dtype=torch.int32, device=DEV), 1, 1, 16)
    cache = hot.KvCache(pool[0], pool[1], torch.tensor([[0, 1], [2, 4]], dtype=torch.int32, device=DEV))
    hot.dlrm_qk_rope_append(plan, x, x, x, torch.empty_like(x), cache, torch.zeros(2, dtype=torch.int32, device=DEV))
    late = hot.QkRope(torch.tensor([8, 2147483647], dtype=torch.int32, device=DEV), 1, 1, 16)
    hot.dlrm_qk_rope_append(late, x, x, x, torch.empty_like(x), cache, torch.ones(2, dtype=torch.int32, device=DEV))   # page 4 of 0..3
    assert not pool.any()


# ------------------------------------------------------------------------------------------------ sequences
RAGGED = [1, 0, 31, 32, 33, 64, 65, 127, 128, 129, 200, 2]
SEQ = [
    # dtype, d, Hq, Hk, lengths of queries, of keys (None: the same items), causal, prefix, slopes, cap, layout
    ("f32", 16, 2, 2, RAGGED, None, True, False, False, 0.0, "packed"),
    ("f32", 72, 6, 3, [1, 257, 0, 90], None, True, True, False, 0.0, "rows"),
    ("f32", 128, 2, 1, [70, 131], None, True, False, True, 20.0, "packed"),
    ("f32", 8, 1, 1, [5, 0, 3], [0, 4, 300], False, False, False, 0.0, "rows"),
    ("f16", 40, 8, 2, [1, 40, 17, 0, 3], [300, 0, 65, 9, 1], False, False, True, 0.0, "packed"),
    ("f16", 64, 4, 1, RAGGED, None, True, True, True, 30.0, "heads"),
    ("f16", 128, 3, 3, [129, 300], None, False, False, False, 0.0, "wide"),
    ("bf16", 64, 4, 4, RAGGED, None, True, False, True, 0.0, "packed"),
    ("bf16", 128, 8, 2, [300, 1, 129], None, True, False, False, 30.0, "packed"),
    ("bf16", 96, 5, 1, [33, 260], [100, 70], True, False, False, 0.0, "heads"),   # new items after cached ones; more queries than keys
    ("bf16", 24, 2, 1, [100, 3, 1], [20, 40, 0], True, True, False, 0.0, "rows"),  # rows that see nothing but a prefix, or nothing
    ("bf16", 128, 16, 1, [1] * 9, [1, 2, 3, 63, 64, 65, 0, 700, 5], True, False, False, 0.0, "rows"),   # one query each
    ("bf16", 56, 2, 2, [0, 0, 1, 0], None, True, False, False, 0.0, "rows"),
    # few rows over many keys
    ("f32", 40, 3, 1, [5, 70, 0], [700, 1300, 90], True, True, True, 20.0, "packed"),
    ("f16", 80, 2, 1, [2, 1, 1, 1], [2694, 513, 0, 20], True, False, True, 0.0, "rows"),
    ("bf16", 64, 4, 2, [600], None, True, False, False, 0.0, "heads"),
    ("f32", 64, 2, 2, [3, 40], [600, 31], False, False, False, 0.0, "rows"),
    ("f32", 88, 3, 3, [3, 40], [600, 1031], False, False, True, 0.0, "rows"),
    ("bf16", 16, 5, 1, [9], [4000], True, False, False, 15.0, "rows"),
    # fp32: many rows, and long walks of not so many
    ("f32", 128, 4, 4, [130] * 70 + [0, 3], None, True, False, True, 0.0, "rows"),
    ("f32", 72, 4, 1, [100, 0, 255] * 60, None, True, True, False, 0.0, "packed"),
    ("f32", 24, 32, 32, [2100, 40, 30], None, True, False, False, 5.0, "rows"),
    ("f32", 96, 32, 16, [1599, 40, 30], None, True, False, False, 0.0, "rows"),
    # no more than one tile of keys
    ("f32", 88, 15, 3, [1, 0, 1, 1, 0] * 20, None, True, False, False, 0.0, "rows"),
    ("f32", 128, 2, 2, [64, 3, 0, 17], None, True, False, True, 0.0, "packed"),
    ("f16", 104, 4, 4, [3, 60, 0, 17], [40, 0, 3, 64], False, False, False, 9.0, "rows"),
]


def seq_case(i, bound=0):
    dtype, d, Hq, Hk, ql, kl, causal, prefix, slopes, cap, where = SEQ[i]
    g, dt = gen(900 + i), DT[dtype]
    kl = ql if kl is None else kl
    qo, ko = ref.offsets(ql), ref.offsets(kl)
    Tq, Tk, B = sum(ql), sum(kl), len(ql)
    q, k, v, do = rand(g, Tq, Hq, d, dtype=dt), rand(g, Tk, Hk, d, dtype=dt), rand(g, Tk, Hk, d, dtype=dt), rand(g, Tq, Hq, d, dtype=dt)
    pre = torch.tensor([(n + 1) // 3 + s % 3 for s, n in enumerate(kl)], dtype=torch.int32) if prefix else None
    sl = torch.tensor([2.0 ** -(1 + h % 8) for h in range(Hq)]) if slopes else None
    up = lambda t: None if t is None else t.to(DEV)
    qd = up(qo)
    seq = hot.SeqBatch(qd, qd if SEQ[i][5] is None else up(ko), Tq, Tk, max(ql) + bound, max(kl) + bound, causal=causal, prefix=up(pre), slopes=up(sl), cap=cap)
    want = ref.attention(q, k, v, qo, ko, causal, pre, sl, d ** -0.5, cap, do)
    return seq, q, k, v, do, where, want


# bound: how much more than the longest sequence the caller says (takes the other way to find a workgroup's sequence)
@pytest.mark.parametrize("bound", [0, 4000])
@pytest.mark.parametrize("i", range(len(SEQ)))
def test_sequence_attention_forward_and_backward(i, bound):
    print("[case]", i, SEQ[i], bound, flush=True)
    seq, q, k, v, do, where, want = seq_case(i, bound)
    (Tq, Hq, d), Hk = q.shape, k.shape[1]
    Q, K, V, DO = (placed(x, where) for x in (q, k, v, do))
    out, dq = (placed(torch.full_like(q, NAN), where) for _ in range(2))
    dk, dv = (placed(torch.full_like(k, NAN), where) for _ in range(2))
    lse = torch.full((Hq, Tq), NAN, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, out, lse)
    ref.close(out, want["out"], want["out_tol"], "out")
    ref.close(lse, want["lse"], want["lse_tol"], "lse")
    ws = hot.alloc_seq_attn_workspace(seq, Hq, Hk, d)
    ws.fill_(255)
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, out, lse, DO, dq, dk, dv, ws)
    for n, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        ref.close(x, want[n], want[n + "_tol"], n)
    again = [torch.empty_like(x) for x in (out, dq, dk, dv)]
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, again[0])                 # without lse; again: bit for bit
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, out, lse, DO, *again[1:], ws)
    for a, b in zip(again, (out, dq, dk, dv)):
        assert torch.equal(a, b)


MANY = [
    # dtype, d, Hq, Hk, sequences, lengths up to, keys up to (None: the same items), causal, prefix, slopes, cap
    ("bf16", 64, 4, 4, 700, 60, None, True, False, True, 0.0),
    ("f16", 40, 8, 2, 500, 40, 700, False, False, False, 0.0),
    ("f16", 32, 6, 2, 900, 33, None, True, True, False, 10.0),
    ("bf16", 96, 4, 2, 800, 50, None, True, False, False, 0.0),
    ("bf16", 128, 16, 4, 14, 600, None, True, True, False, 30.0),
    ("bf16", 128, 16, 2, 14, 600, None, True, False, True, 0.0),
    ("f16", 72, 12, 12, 16, 700, None, True, False, False, 0.0),
    ("f32", 96, 8, 4, 24, 700, None, True, False, False, 0.0),
    ("f32", 128, 16, 2, 14, 600, None, True, False, True, 0.0),
    ("f32", 24, 4, 2, 700, 60, None, True, True, False, 20.0),
    ("f32", 120, 4, 4, 900, 40, None, True, False, False, 0.0),
    ("bf16", 112, 8, 1, 600, 40, 20, False, False, False, 0.0),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_many_rows(i):
    """Enough rows for the kernels that big batches take, short and long sequences, some without items."""
    print("[case]", i, MANY[i], flush=True)
    dtype, d, Hq, Hk, B, top, ktop, causal, prefix, slopes, cap = MANY[i]
    rng, g, dt = np.random.RandomState(i), gen(1200 + i), DT[dtype]
    ql = rng.randint(0, top + 1, B)
    ql[:2] = top, 0
    kl = ql if ktop is None else rng.randint(0, ktop + 1, B)
    qo, ko = ref.offsets(ql), ref.offsets(kl)
    Tq, Tk = int(ql.sum()), int(kl.sum())
    q, k, v, do = (rand(g, T, H, d, dtype=dt) for T, H in ((Tq, Hq), (Tk, Hk), (Tk, Hk), (Tq, Hq)))
    pre = torch.tensor(kl // 4, dtype=torch.int32) if prefix else None
    sl = torch.tensor([2.0 ** -(1 + h % 8) for h in range(Hq)]) if slopes else None
    up = lambda t: None if t is None else t.to(DEV)
    seq = hot.SeqBatch(up(qo), up(ko), Tq, Tk, int(ql.max()), int(kl.max()), causal=causal, prefix=up(pre), slopes=up(sl), cap=cap)
    Q, K, V, DO = (up(x) for x in (q, k, v, do))
    out, dq, dk, dv = (torch.full_like(x, NAN) for x in (Q, Q, K, V))
    lse = torch.full((Hq, Tq), NAN, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, out, lse)
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, out, lse, DO, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
    want = ref.attention(q, k, v, qo, ko, causal, pre, sl, d ** -0.5, cap, do)
    for n, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.close(x, want[n], want[n + "_tol"], n)


def test_long_sequences():
    """Many tiles, an uneven end, shared heads; against the formula in 64 bits on the device."""
    g = torch.Generator(device=DEV).manual_seed(3)
    n, Hq, Hk, d = 2500, 4, 2, 128
    for dt in (torch.bfloat16, torch.float32):
        q, do = (torch.randn(n, Hq, d, generator=g, device=DEV).to(dt) for _ in range(2))
        k, v = (torch.randn(n, Hk, d, generator=g, device=DEV).to(dt) for _ in range(2))
        off = torch.tensor([0, n], device=DEV)
        seq = hot.SeqBatch(off, off, n, n, n, n)
        want = ref.attention(*(x.cpu() for x in (q, k, v)), off.cpu(), off.cpu(), True, None, None, d ** -0.5, 0.0, do.cpu())
        out, dq, dk, dv = (torch.empty_like(x) for x in (q, q, k, v))
        lse = torch.empty(Hq, n, device=DEV)
        hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
        hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
        for name, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
            ref.close(x, want[name], want[name + "_tol"], name)


def test_scores_far_apart():
    """Scores of +-1e4: the softmax is one-hot, and nothing overflows on the way."""
    n, d = 70, 32
    g = gen(5)
    q, k, v = (rand(g, n, 1, d, scale=s) for s in (100.0, 300.0, 1.0))
    off = torch.tensor([0, n], device=DEV)
    out, lse = torch.empty(n, 1, d, device=DEV), torch.empty(1, n, device=DEV)
    hot.dlrm_seq_attn_fwd(hot.SeqBatch(off, off, n, n, n, n, scale=1.0), q.to(DEV), k.to(DEV), v.to(DEV), out, lse)
    want = ref.attention(q, k, v, off.cpu(), off.cpu(), True, None, None, 1.0, 0.0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    ref.close(lse, want["lse"], want["lse_tol"], "lse")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_what_lies_outside_a_sequence_has_no_part(dtype):
    """Neighbours full of NaN and infinity leave a sequence's own results as they are."""
    dt, g, d, H = DT[dtype], gen(11), 64, 2
    lens = [45, 77, 30]
    off = ref.offsets(lens)
    x = [rand(g, sum(lens), H, d, dtype=dt) for _ in range(4)]
    def run(x):
        q, k, v, do = (t.to(DEV) for t in x)
        o = off.to(DEV)
        seq = hot.SeqBatch(o, o, sum(lens), sum(lens), max(lens), max(lens))
        out, dq, dk, dv = (torch.empty_like(q) for _ in range(4))
        lse = torch.empty(H, sum(lens), device=DEV)
        hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
        hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, H, H, d))
        return [t[45:122].clone() for t in (out, dq, dk, dv)]
    clean = run(x)
    for t in x:
        t[:45], t[122:] = NAN, math.inf
    for a, b in zip(clean, run(x)):
        assert torch.equal(a, b)


def test_gradients_against_differences():
    """<grad, step> against central differences of the forward itself, in fp32, all masks and scores at once."""
    g, d, Hq, Hk = gen(21), 24, 4, 2
    lens = [19, 1, 40]
    off, T = ref.offsets(lens).to(DEV), sum(lens)
    pre = torch.tensor([4, 0, 9], dtype=torch.int32, device=DEV)
    sl = torch.tensor([0.5, 0.25, 0.125, 0.0625], device=DEV)
    seq = hot.SeqBatch(off, off, T, T, 40, 40, prefix=pre, slopes=sl, cap=3.0)
    x = [rand(g, T, H, d).to(DEV) for H in (Hq, Hk, Hk)]
    do = rand(g, T, Hq, d).to(DEV)
    def f(y):
        out = torch.empty(T, Hq, d, device=DEV)
        lse = torch.empty(Hq, T, device=DEV)
        hot.dlrm_seq_attn_fwd(seq, *y, out, lse)
        return out, lse
    out, lse = f(x)
    grads = [torch.empty_like(t) for t in x]
    hot.dlrm_seq_attn_bwd(seq, *x, out, lse, do, *grads, hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
    eps = 2.0 ** -7
    for j in range(3):
        step = rand(g, *x[j].shape).to(DEV)
        up, down = (f([t + s * eps * step if i == j else t for i, t in enumerate(x)])[0].double() for s in (1, -1))
        slope = float(((up - down) * do.double()).sum() / (2 * eps))
        mine = float((grads[j].double() * step.double()).sum())
        # third-order term: eps^2 / 6 times a third derivative of the size of the sum's terms; fp32: 2^-22 |out||do| / eps
        size = float((grads[j].double().abs() * step.double().abs()).sum())
        assert abs(slope - mine) <= 2e-3 * size, (j, slope, mine, size)


def test_another_stream_and_other_tensors_of_the_same_plan():
    g, d, H, n = gen(31), 32, 2, 50
    off = torch.tensor([0, 20, n], device=DEV)
    seq = hot.SeqBatch(off, off, n, n, 30, 30)
    a, b = ([rand(g, n, H, d, dtype=torch.bfloat16).to(DEV) for _ in range(3)] for _ in range(2))
    out = [torch.empty(n, H, d, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    hot.dlrm_seq_attn_fwd(seq, *a, out[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        hot.dlrm_seq_attn_fwd(seq, *b, out[1])
        hot.dlrm_seq_attn_fwd(seq, *a, out[2])
    s.synchronize()
    assert torch.equal(out[0], out[2]) and not torch.equal(out[0], out[1])


# ------------------------------------------------------------------------------------------------ the cache
CACHE = [
    # dtype, d, Hq, Hk, page, lengths, max_len, slopes, cap
    ("f32", 16, 2, 2, 16, [0, 1, 15, 16, 17, 200], 200, False, 0.0),
    ("f32", 128, 8, 1, 8, [3, 700, 0], 700, True, 30.0),
    ("f32", 72, 6, 3, 1, [40, 5], 64, False, 0.0),
    ("f16", 40, 8, 2, 32, [1, 31, 32, 33, 65, 3000], 3000, True, 0.0),
    ("f16", 64, 5, 1, 64, [900], 900, False, 5.0),
    ("bf16", 128, 16, 4, 64, [5000], 5000, False, 0.0),
    ("bf16", 128, 16, 4, 32, [1, 0, 129, 2047, 256], 2500, True, 50.0),
    ("bf16", 64, 40, 1, 16, [77, 300], 300, False, 0.0),      # more heads to a key head than one tile has columns
    ("bf16", 8, 1, 1, 1024, [2000, 1], 2048, False, 0.0),
    ("bf16", 96, 17, 1, 128, [130] * 3, 130, True, 0.0),
    ("bf16", 32, 4, 4, 16, [-3, 50, 70], 60, False, 0.0),     # below nothing, and above the bound
]


@pytest.mark.parametrize("i", range(len(CACHE)))
def test_cache_attention(i):
    print("[case]", i, CACHE[i], flush=True)
    dtype, d, Hq, Hk, page, lens, max_len, slopes, cap = CACHE[i]
    g, dt, B = gen(300 + i), DT[dtype], len(lens)
    cols = (max(max_len, max(lens)) + page - 1) // page
    n_pages = B * cols + 2
    table = torch.randperm(n_pages, generator=g)[:B * cols].view(B, cols).to(torch.int32)
    pool_k, pool_v = (torch.full((n_pages, Hk, page, d), NAN, dtype=dt) for _ in range(2))    # whatever is past a length is NaN
    q = rand(g, B, Hq, d, dtype=dt)
    eff = [max(0, min(n, max_len)) for n in lens]
    k, v = (rand(g, sum(eff), Hk, d, dtype=dt) for _ in range(2))
    off = ref.offsets(eff)
    for s, n in enumerate(eff):
        for p in range(n):
            pool_k[table[s, p // page], :, p % page] = k[int(off[s]) + p]
            pool_v[table[s, p // page], :, p % page] = v[int(off[s]) + p]
    sl = torch.tensor([2.0 ** -(1 + h % 8) for h in range(Hq)]) if slopes else None
    want = ref.attention(q, k, v, torch.arange(B + 1), off, False, None, sl, d ** -0.5, cap)
    cache = hot.KvCache(pool_k.to(DEV), pool_v.to(DEV), table.to(DEV))
    Q = placed(q, "packed")
    out = placed(torch.full_like(q, NAN), "packed")
    L = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = hot.alloc_cache_attn_workspace(cache, Hq, max_len)
    ws.fill_(255)
    hot.dlrm_cache_attn(cache, L, max_len, Q, out, ws, slopes=None if sl is None else sl.to(DEV), cap=cap)
    ref.close(out, want["out"], want["out_tol"], "out")
    again = torch.empty(B, Hq, d, dtype=dt, device=DEV)
    hot.dlrm_cache_attn(cache, L, max_len, Q, again, ws, slopes=None if sl is None else sl.to(DEV), cap=cap)
    assert torch.equal(out, again)


def test_pages_that_are_not_there_take_no_part():
    g, d, page = gen(8), 32, 16
    k, v = (rand(g, 6, 1, page, d) for _ in range(2))
    q = rand(g, 1, 1, d)
    table = torch.tensor([[4, -1, 2, 6, 0]], dtype=torch.int32)      # 6 pages: 6 is none
    cache = hot.KvCache(k.to(DEV), v.to(DEV), table.to(DEV))
    out = torch.empty(1, 1, d, device=DEV)
    hot.dlrm_cache_attn(cache, torch.tensor([70], dtype=torch.int32, device=DEV), 80, q.to(DEV), out, hot.alloc_cache_attn_workspace(cache, 1, 80))
    K, V = torch.cat([k[4, 0], k[2, 0], k[0, 0, :6]])[:, None], torch.cat([v[4, 0], v[2, 0], v[0, 0, :6]])[:, None]
    want = ref.attention(q, K, V, torch.tensor([0, 1]), torch.tensor([0, 38]), False, None, None, d ** -0.5, 0.0)
    ref.close(out, want["out"], want["out_tol"], "out")


def test_offsets_past_32_bits_in_a_long_cache():
    """5 GB of keys: rows whose byte offset needs 33 bits are read, and stored by the append, at their place."""
    d, page, Hk = 128, 64, 4
    n_pages = 80000
    pool = torch.zeros(2, n_pages, Hk, page, d, dtype=torch.bfloat16, device=DEV)
    table = torch.tensor([[n_pages - 1, 3]], dtype=torch.int32, device=DEV)
    cache = hot.KvCache(pool[0], pool[1], table)
    g = gen(4)
    T = 100
    q, k, v = (rand(g, T, H, d, dtype=torch.bfloat16) for H in (8, Hk, Hk))
    plan = hot.QkRope(torch.arange(T, dtype=torch.int32, device=DEV), 8, Hk, d)
    hot.dlrm_qk_rope_append(plan, q.to(DEV), k.to(DEV), v.to(DEV), torch.empty(T, 8, d, dtype=torch.bfloat16, device=DEV), cache,
                            torch.zeros(T, dtype=torch.int32, device=DEV))
    assert torch.equal(pool[1, n_pages - 1].cpu(), v[:64].transpose(0, 1)) and torch.equal(pool[0, 3, :, :36].cpu(), k[64:].transpose(0, 1))
    assert int((pool[0] != 0).any(-1).sum()) == T * Hk
    out = torch.empty(1, 8, d, dtype=torch.bfloat16, device=DEV)
    hot.dlrm_cache_attn(cache, torch.tensor([T], dtype=torch.int32, device=DEV), 128, q[-1:].to(DEV), out, hot.alloc_cache_attn_workspace(cache, 8, 128))
    want = ref.attention(q[-1:], k, v, torch.tensor([0, 1]), torch.tensor([0, T]), False, None, None, d ** -0.5, 0.0)
    ref.close(out, want["out"], want["out_tol"], "out")


def test_calls_in_a_graph_replay_like_eager_calls():
    """Forward, backward and cached attention captured once, replayed over new inputs between eager work."""
    g, d, Hq, Hk = gen(77), 64, 4, 2
    lens = [40, 3, 130]
    off, T = ref.offsets(lens).to(DEV), sum(lens)
    seq = hot.SeqBatch(off, off, T, T, 130, 130)
    mk = lambda H: torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV)
    q, k, v, do, out, dq, dk, dv = (mk(H) for H in (Hq, Hk, Hk, Hq, Hq, Hq, Hk, Hk))
    lse, ws = torch.empty(Hq, T, device=DEV), hot.alloc_seq_attn_workspace(seq, Hq, Hk, d)
    pool = torch.zeros(2, 64, Hk, 16, d, dtype=torch.bfloat16, device=DEV)
    cache = hot.KvCache(pool[0], pool[1], torch.arange(60, dtype=torch.int32, device=DEV).view(3, 20))
    L, cout = torch.tensor([300, 17, 1], dtype=torch.int32, device=DEV), torch.empty(3, Hq, d, dtype=torch.bfloat16, device=DEV)
    cws = hot.alloc_cache_attn_workspace(cache, Hq, 320)

    def step():
        hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
        hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, ws)
        hot.dlrm_cache_attn(cache, L, 320, q[:3], cout, cws)

    def fill():
        for x in (q, k, v, do, pool):
            x.copy_(rand(g, *x.shape, dtype=torch.bfloat16))
    fill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        fill()
        graph.replay()
        got = [x.clone() for x in (out, lse, dq, dk, dv, cout)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, dq, dk, dv, cout)):
            assert torch.equal(a, b)


def test_the_sequence_encoder_learns_and_its_cache_agrees():
    """examples/history_encoder.py: lookup, projections, norm and rotation, attention, the way back, the row update, and the cache."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import history_encoder
    losses, off = history_encoder.main(["--steps", "12", "--users", "64", "--items", "500"])
    assert all(math.isfinite(x) for x in losses) and losses[-1] < 0.97 * losses[0]
    assert off < 1e-5
