"""Attention of one new item with a learned bias (dlrm_cache_attn_bias), and of several new items (dlrm_cache_tree_attn), over a paged cache, against
a plain 64-bit form (bias_ref), with elementwise bounds."""
import math
import random

import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from history_ref import close, offsets
from test_gpu_relative_bias import DEV, DT, NAN, bounds_of, gen, placed, rand

pytestmark = pytest.mark.gpu


class Paged:
    """Sequences of `lens` items in pages handed out in random order; what no sequence holds is NaN."""

    def __init__(self, g, lens, cols, page, Hk, d, dt, missing=()):
        B, self.lens, self.page = len(lens), lens, page
        n = max(1, sum(-(-m // page) for m in lens))
        self.k, self.v = ([rand(g, m, Hk, d, dtype=dt) for m in lens] for _ in range(2))
        self.pool = torch.full((2, n + 1, Hk, page, d), NAN, dtype=dt)
        table = torch.full((B, cols), -1, dtype=torch.int32)
        free = torch.randperm(n + 1, generator=g).tolist()
        self.gone = [torch.zeros(m, dtype=torch.bool) for m in lens]
        for s, m in enumerate(lens):
            for p in range(-(-m // page)):
                at, I = free.pop(), slice(p * page, min(m, (p + 1) * page))
                if (s, p) in missing:
                    table[s, p] = [-5, n + 1, 2 ** 31 - 1][p % 3]
                    self.gone[s][I] = True
                    continue
                table[s, p] = at
                for x, y in zip(self.pool, (self.k, self.v)):
                    x[at, :, :I.stop - I.start] = y[s][I].transpose(0, 1)
        self.dev = self.pool.to(DEV)
        self.cache = hot.KvCache(self.dev[0], self.dev[1], table.to(DEV))
        self.dlens = torch.tensor(lens, dtype=torch.int32, device=DEV)


def up(x):
    return None if x is None else x.to(DEV)


ONE = [
    # type, query heads, key heads, d, page, lengths, slopes, cap, buckets, bounds, where the rows lie
    ("f32", 4, 4, 64, 16, [1, 200, 0, 33, 64], False, 0.0, 32, "log", "rows"),
    ("f32", 6, 2, 72, 8, [5000, 17], True, 0.0, 33, "one by one", "packed"),
    ("bf16", 16, 4, 128, 32, [1, 8000, 300, 2047], False, 50.0, 64, "log", "packed"),
    ("bf16", 33, 1, 24, 64, [700, 90], False, 0.0, 128, "one by one", "heads"),
    ("bf16", 2, 2, 8, 1, [1000, 31], False, 0.0, 5, "edges", "wide"),
    ("f16", 8, 2, 40, 128, [0, 1000, 257], False, 0.0, 1, None, "rows"),
    ("f16", 5, 1, 96, 16, [40000], False, 0.0, 100, "log", "rows"),
    ("f16", 4, 2, 64, 16, [300, 20], False, 300.0, 9, "one by one", "rows"),
]


@pytest.mark.parametrize("i", range(len(ONE)))
def test_one_new_item_with_a_bias(i):
    dt, Hq, Hk, d, page, lens, slopes, cap, n, kind, where = ONE[i]
    print("[case]", i, ONE[i], flush=True)
    g, dt, B, top = gen(300 + i), DT[dt], len(lens), max(lens)
    cols = -(-top // page) + 1
    c = Paged(g, lens, cols, page, Hk, d, dt)
    q = rand(g, B, Hq, d, dtype=dt)
    table, bounds = rand(g, Hq, n), bounds_of(kind, n)
    sl = torch.rand(Hq, generator=g) * 0.1 if slopes else None
    out = placed(torch.full_like(q, NAN), where)
    ws = hot.alloc_cache_attn_bias_workspace(c.cache, Hq, top)
    ws.fill_(255)
    hot.dlrm_cache_attn_bias(c.cache, c.dlens, top, hot.RelBias(table.to(DEV), up(bounds)), placed(q, where), out, ws, slopes=up(sl), cap=cap)
    for s, m in enumerate(lens):
        want, tol = ref.cached(q[s:s + 1], c.k[s], c.v[s], None, None, torch.tensor([m - 1]), None, sl, table, bounds, d ** -0.5, cap)
        close(out[s:s + 1], want, tol, "sequence %d" % s)


def tree_of(g, n, kind):
    """(last, depth)"""
    if kind == "flat":
        return list(range(n)), [0] * n
    if kind in ("chain", "none"):
        return [n - 1] * n, list(range(n))
    if kind == "far apart":   # places all over, as of items whose distances are not what they stand behind
        return list(range(n)), torch.randint(0, 900, (n,), generator=g).tolist()
    if kind == "hidden":   # nobody sees the odd ones
        return [j - 1 if j % 2 else n - 1 for j in range(n)], list(range(n))
    rng = random.Random(int(torch.randint(1 << 30, (1,), generator=g)))
    return hot.tree_order([rng.randrange(max(-1, i - 5), i) for i in range(n)])[1:]


TREES = [
    # type, query heads, key heads, d, page, lengths, new items, shape, slopes, cap, buckets (0: no bias), bounds, where the rows lie
    ("f32", 2, 1, 16, 8, [0, 5, 40], [1, 3, 0], "tree", False, 0.0, 0, None, "rows"),
    ("f32", 6, 3, 72, 8, [1500, 1, 77, 0], [70, 129, 1, 33], "chain", False, 0.0, 16, "log", "packed"),
    ("f32", 8, 2, 128, 64, [300, 64, 2000], [9, 8, 20], "tree", True, 20.0, 33, "one by one", "heads"),
    ("f32", 1, 1, 32, 16, [0, 0, 3], [5, 60, 2], "flat", False, 0.0, 0, None, "wide"),
    ("bf16", 8, 2, 64, 64, [1, 200, 90, 64], [8, 8, 8, 8], "tree", False, 0.0, 0, None, "packed"),
    ("bf16", 16, 4, 128, 32, [5000, 1, 700], [60, 30, 1], "tree", False, 50.0, 64, "log", "packed"),
    ("bf16", 4, 4, 128, 16, [33, 257], [7, 15], "none", True, 0.0, 0, None, "rows"),
    ("bf16", 16, 4, 96, 16, [9000], [64], "tree", False, 0.0, 0, None, "rows"),
    ("bf16", 33, 1, 24, 8, [100, 31], [2, 5], "tree", False, 0.0, 128, "one by one", "wide"),
    ("bf16", 80, 1, 16, 8, [40, 2], [3, 1], "hidden", False, 0.0, 6, "one by one", "rows"),
    ("bf16", 2, 2, 8, 1, [64, 7, 0], [1, 40, 4], "hidden", False, 0.0, 0, None, "rows"),
    ("f16", 8, 2, 40, 16, [0, 1000, 333, 8], [40, 1, 17, 2], "flat", True, 0.0, 0, None, "packed"),
    ("f16", 5, 1, 104, 128, [20000, 50], [13, 14], "tree", False, 0.0, 20, "both", "heads"),
    ("f16", 4, 2, 64, 16, [130, 20], [40, 65], "chain", False, 300.0, 5, "edges", "rows"),
    ("f16", 4, 1, 128, 64, [1025, 3], [200, 100], "none", False, 0.0, 5, "far", "rows"),
    ("bf16", 33, 1, 128, 16, [300, 45, 17], [8, 3, 1], "tree", False, 0.0, 128, "one by one", "rows"),   # the most biases in LDS: 33 heads of 128
    ("f32", 64, 1, 96, 16, [200, 31], [2, 3], "chain", False, 0.0, 128, "log", "packed"),
    ("bf16", 4, 2, 64, 32, [3000, 2000], [90, 70], "far apart", False, 0.0, 30, "log", "rows"),          # places too far from each other for one window
    ("f32", 2, 2, 32, 8, [400, 20], [12, 5], "far apart", True, 0.0, 30, "log", "rows"),
    ("bf16", 8, 4, 128, 64, [700, 64], [130, 33], "tree", False, 15.0, 40, "log", "heads"),
]


def tree_case(i):
    dt, Hq, Hk, d, page, lens, new, kind, slopes, cap, n, bk, where = TREES[i]
    print("[case]", i, TREES[i], flush=True)
    g, dt, T = gen(600 + i), DT[dt], sum(new)
    c = Paged(g, lens, max(1, -(-max(lens) // page)), page, Hk, d, dt, missing=((1, 1),) if i % 4 == 1 else ())
    shapes = [tree_of(g, m, kind) for m in new]
    last = torch.tensor(sum((list(x[0]) for x in shapes), []), dtype=torch.int32)
    pos = torch.tensor(sum(([m + y for y in x[1]] for m, x in zip(lens, shapes)), []), dtype=torch.int32)
    x = {"q": rand(g, T, Hq, d, dtype=dt), "k": rand(g, T, Hk, d, dtype=dt), "v": rand(g, T, Hk, d, dtype=dt)}
    table, bounds = (rand(g, Hq, n), bounds_of(bk, n)) if n else (None, None)
    sl = torch.rand(Hq, generator=g) * 0.1 if slopes else None
    bias = hot.RelBias(table.to(DEV), up(bounds)) if n else None
    items = hot.NewItems(offsets(new).to(DEV), T, max(new), last=None if kind == "none" else last.to(DEV), positions=pos.to(DEV) if n or slopes else None)
    return g, c, new, x, (pos, last, sl, table, bounds, d ** -0.5, cap), items, bias, up(sl), where


def run_tree(c, x, items, bias, slopes, cap, where, top=None, dlens=None):
    top = max(c.lens) if top is None else top
    out = placed(torch.full_like(x["q"], NAN), where)
    ws = hot.alloc_cache_tree_attn_workspace(c.cache, x["q"].shape[1], top, items)
    ws.fill_(255)   # (NaN, whatever is read of it before it is written)
    hot.dlrm_cache_tree_attn(c.cache, c.dlens if dlens is None else dlens, top, items, *(placed(x[n], where) for n in "qkv"), out, ws, bias=bias, slopes=slopes,
                             cap=cap)
    return out


def check_tree(c, new, x, how, out, lens=None):
    pos, last, *score = how
    at = 0
    for s, m in enumerate(c.lens if lens is None else lens):
        I, keep = slice(at, at + new[s]), ~c.gone[s][:m]
        at = I.stop
        if not new[s]:
            continue
        if not keep.all():   # pages that are not there: their keys are not seen
            want, tol = gone_pages(c, s, x, I, pos, last, score)
        else:
            want, tol = ref.cached(x["q"][I], c.k[s][:m], c.v[s][:m], x["k"][I], x["v"][I], pos[I], last[I], *score)
        close(out[I], want, tol, "sequence %d" % s)


def gone_pages(c, s, x, I, pos, last, score):
    """The cached items that are left, at the places that they have: as new items in front of the others, which all of those see."""
    sl, table, bounds, scale, cap = score
    keep = torch.nonzero(~c.gone[s])[:, 0]
    n, old = I.stop - I.start, len(keep)
    q = torch.cat([torch.zeros(old, *x["q"].shape[1:], dtype=x["q"].dtype), x["q"][I]])
    k, v = (torch.cat([y[s][keep], x[m][I]]) for y, m in ((c.k, "k"), (c.v, "v")))
    p = torch.cat([keep.int(), pos[I]])
    l = torch.cat([torch.full((old,), old + n - 1, dtype=torch.int32), last[I] + old])
    none = k[:0]
    want, tol = ref.cached(q, none, none, k, v, p, l, sl, table, bounds, scale, cap)
    return want[old:], tol[old:]


@pytest.mark.parametrize("i", range(len(TREES)))
def test_new_items_over_the_cache_and_one_another(i):
    g, c, new, x, how, items, bias, sl, where = tree_case(i)
    cap = how[-1]
    out = run_tree(c, x, items, bias, sl, cap, where)
    check_tree(c, new, x, how, out)
    before = c.dev.clone()
    again = run_tree(c, x, items, bias, sl, cap, where)
    assert torch.equal(out.nan_to_num(), again.nan_to_num()) and torch.equal(before.nan_to_num(), c.dev.nan_to_num())   # the cache is not written
    assert not torch.isnan(out).any()


@pytest.mark.parametrize("i", [4, 5, 11])
def test_lengths_above_the_bound_count_as_the_bound(i):
    g, c, new, x, how, items, bias, sl, where = tree_case(i)
    top = max(c.lens) // 2
    out = run_tree(c, x, items, bias, sl, how[-1], where, top=top)
    check_tree(c, new, x, how, out, lens=[min(m, top) for m in c.lens])
    # negative lengths are empty caches, with a bound of none too
    dlens = torch.full_like(c.dlens, -3)
    for bound in (top, 0):
        out = run_tree(c, x, items, bias, sl, how[-1], where, top=bound, dlens=dlens)
        check_tree(c, new, x, how, out, lens=[0] * len(c.lens))


def test_items_past_the_bound_are_neither_answered_nor_seen():
    g, c, new, x, how, items, bias, sl, where = tree_case(4)
    few = hot.NewItems(items.off, items.T, 5, last=items.last)
    out = run_tree(c, x, few, bias, sl, 0.0, "rows")
    want = run_tree(c, x, items, bias, sl, 0.0, "rows")
    part = (torch.arange(items.T) % 8 < 5).to(DEV)
    close(out[part], want[part].double().cpu(), 2 ** -7 * want[part].double().abs().cpu() + 1e-3, "items")
    assert torch.isnan(out[~part]).all()


def test_loose_bounds_and_rows_behind_the_last_item():
    """max_items above all that there are; rows behind the batch's own stay as they were."""
    g, c, new, x, how, items, bias, sl, where = tree_case(5)
    loose = hot.NewItems(items.off, items.T, 2 ** 31 - 1, last=items.last, positions=items.positions)
    out = run_tree(c, x, loose, bias, sl, how[-1], "rows", top=1 << 20)
    check_tree(c, new, x, how, out)
    more = torch.full((items.T + 3, *x["q"].shape[1:]), 7.0, dtype=x["q"].dtype, device=DEV)
    dev = {n: t.to(DEV) for n, t in x.items()}
    hot.dlrm_cache_tree_attn(c.cache, c.dlens, 5000, items, dev["q"], dev["k"], dev["v"], more[:items.T],
                             hot.alloc_cache_tree_attn_workspace(c.cache, 16, 5000, items), bias=bias, cap=how[-1])
    check_tree(c, new, x, how, more[:items.T])
    assert (more[items.T:] == 7).all()


def test_no_items_at_all():
    c = Paged(gen(1), [5, 9], 2, 8, 2, 16, torch.float32)
    none = hot.NewItems(torch.zeros(3, dtype=torch.int64, device=DEV), 0, 4)
    x = [torch.empty(0, H, 16, device=DEV) for H in (4, 2, 2, 4)]
    hot.dlrm_cache_tree_attn(c.cache, c.dlens, 9, none, *x, None)
    torch.cuda.synchronize()


def test_one_item_with_no_cache_is_its_own_value():
    g = gen(2)
    c = Paged(g, [0, 0], 1, 8, 2, 32, torch.bfloat16)
    items = hot.NewItems(torch.tensor([0, 1, 2], device=DEV), 2, 1)
    x = {n: rand(g, 2, H, 32, dtype=torch.bfloat16) for n, H in (("q", 6), ("k", 2), ("v", 2))}
    assert torch.equal(run_tree(c, x, items, None, None, 0.0, "rows", top=0).cpu(), x["v"].repeat_interleave(3, 1))


def test_a_chain_over_the_cache_is_the_whole_history():
    """A prompt run piece by piece: each piece over the cache of the pieces before it, then appended, against the history run at once; and its newest item
    alone (dlrm_cache_attn_bias) once it is in the cache."""
    g, Hq, Hk, d, page = gen(3), 8, 2, 64, 16
    lens, B = [150, 37, 64], 3
    off, T = offsets(lens), sum(lens)
    q, k, v = (rand(g, T, H, d, dtype=torch.bfloat16).to(DEV) for H in (Hq, Hk, Hk))
    bias = hot.RelBias(torch.randn(Hq, 32, device=DEV), hot.relative_bounds(32, 100, device=DEV))
    users = torch.repeat_interleave(torch.arange(B), torch.tensor(lens)).to(torch.int32)
    pos = (torch.arange(T) - off[users.long()]).to(torch.int32)
    rope = lambda at: hot.QkRope(pos[at].to(DEV), Hq, Hk, d, inv_freq=hot.rope_frequencies(d, device=DEV))
    qr, kr, whole = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    hot.dlrm_qk_rope_fwd(rope(slice(None)), q, k, qr, kr)
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 150, 150)
    hot.dlrm_seq_attn_bias_fwd(seq, bias, qr, kr, v, whole)
    pool = torch.full((2, 60, Hk, page, d), NAN, dtype=torch.bfloat16, device=DEV)
    cache = hot.KvCache(pool[0], pool[1], torch.randperm(60, generator=g).to(torch.int32).view(3, 20).to(DEV))
    got, done = torch.full_like(q, NAN), [0, 0, 0]
    while done != lens:
        take = [min(n - m, 41) for n, m in zip(lens, done)]
        at = torch.cat([torch.arange(int(off[s]) + done[s], int(off[s]) + done[s] + take[s]) for s in range(B)])
        items = hot.NewItems(offsets(take).to(DEV), sum(take), max(take), positions=pos[at].to(DEV))
        a = at.to(DEV)
        x, y, z, o = qr[a], kr[a], v[a], torch.empty_like(q[a])
        dl = torch.tensor(done, dtype=torch.int32, device=DEV)
        hot.dlrm_cache_tree_attn(cache, dl, max(done), items, x, y, z, o, hot.alloc_cache_tree_attn_workspace(cache, Hq, max(done), items), bias=bias)
        got[a] = o
        hot.dlrm_qk_rope_append(rope(at), q[a], k[a], v[a], torch.empty_like(x), cache, users[at].to(DEV))
        done = [m + n for m, n in zip(done, take)]
    # both are the bf16 of one number, fp32's errors and weights rounded once apart
    limit = (2 ** -7 * whole.double().abs() + 2 ** -8 * v.double().abs().max()).cpu()
    close(got, whole.double().cpu(), limit, "pieces")
    newest, o = (off[1:] - 1).to(DEV), torch.empty(B, Hq, d, dtype=torch.bfloat16, device=DEV)
    hot.dlrm_cache_attn_bias(cache, torch.tensor(lens, dtype=torch.int32, device=DEV), 150, bias, qr[newest], o,
                             hot.alloc_cache_attn_bias_workspace(cache, Hq, 150))
    close(o, whole[newest].double().cpu(), limit[newest.cpu()], "newest")


def test_one_item_without_a_bias_is_the_unbiased_attention():
    """dlrm_cache_attn, whose newest item is in the cache, and the same item as a new one beside the cache; fp32, sums in another order."""
    g, lens = gen(4), [700, 1, 40]
    c = Paged(g, lens, 50, 16, 2, 64, torch.float32)
    q = rand(g, 3, 8, 64)
    a, b = (torch.empty(3, 8, 64, device=DEV) for _ in range(2))
    hot.dlrm_cache_attn(c.cache, c.dlens, 700, q.to(DEV), a, hot.alloc_cache_attn_workspace(c.cache, 8, 700))
    items = hot.NewItems(torch.arange(4, device=DEV), 3, 1)
    k, v = (torch.stack([y[s][-1] for s in range(3)]).to(DEV) for y in (c.k, c.v))
    hot.dlrm_cache_tree_attn(c.cache, c.dlens - 1, 699, items, q.to(DEV), k, v, b, hot.alloc_cache_tree_attn_workspace(c.cache, 8, 699, items))
    assert float((a - b).abs().max()) < 1e-5


def test_values_of_other_sequences_and_pages_do_not_matter():
    """(the pool's unused places, and those past a sequence's end, are NaN in every test here) Infinities in another sequence's rows reach none of this one's."""
    g, c, new, x, how, items, bias, sl, where = tree_case(6)
    one = run_tree(c, x, items, bias, sl, 0.0, "rows")
    for n in "kv":
        x[n][7:] = math.inf
    x["q"][7:] = NAN
    two = run_tree(c, x, items, bias, sl, 0.0, "rows")
    assert torch.equal(one[:7], two[:7])


def test_more_sequences_than_one_launch_of_the_join_takes():
    """70000 sequences of one item, pages of one item each and a bound on the length that more than one chunk's pages hold."""
    B, d = 70000, 8
    cache = hot.KvCache(torch.randn(4, 1, 1, d, device=DEV), torch.randn(4, 1, 1, d, device=DEV), torch.zeros(B, 1100, dtype=torch.int32, device=DEV))
    q, k, v, out = (torch.randn(B, 1, d, device=DEV) for _ in range(4))
    items = hot.NewItems(torch.arange(B + 1, device=DEV), B, 1)
    lens = torch.ones(B, dtype=torch.int32, device=DEV)
    ws = hot.alloc_cache_tree_attn_workspace(cache, 1, 1100, items)
    assert ws.numel() >= B * 2 * (d + 2) * 4
    hot.dlrm_cache_tree_attn(cache, lens, 1100, items, q, k, v, out, ws)
    a = (q * cache.k[0, 0, 0]).sum(-1, keepdim=True) * d ** -0.5
    b = (q * k).sum(-1, keepdim=True) * d ** -0.5
    w = torch.sigmoid(b - a)
    assert float((out - (w * v + (1 - w) * cache.v[0, 0, 0])).abs().max()) < 1e-5


def test_a_graph_of_calls_over_the_cache_replays_like_eager_calls():
    g, Hq, Hk, d = gen(9), 8, 2, 64
    c = Paged(g, [300, 17, 1], 20, 16, Hk, d, torch.bfloat16)
    new, T = [6, 1, 9], 16
    last = torch.tensor(sum((tree_of(g, m, "tree")[0] for m in new), []), dtype=torch.int32, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) + 300
    items = hot.NewItems(offsets(new).to(DEV), T, 9, last=last, positions=pos)
    bias = hot.RelBias(torch.randn(Hq, 20, device=DEV), hot.relative_bounds(20, 100, device=DEV))
    q, k, v, out = (torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV) for H in (Hq, Hk, Hk, Hq))
    one = torch.empty(3, Hq, d, dtype=torch.bfloat16, device=DEV)
    ws, ws1 = hot.alloc_cache_tree_attn_workspace(c.cache, Hq, 320, items), hot.alloc_cache_attn_bias_workspace(c.cache, Hq, 320)

    def step():
        hot.dlrm_cache_tree_attn(c.cache, c.dlens, 320, items, q, k, v, out, ws, bias=bias)
        hot.dlrm_cache_attn_bias(c.cache, c.dlens, 320, bias, q[:3], one, ws1)

    def fill():
        for x in (q, k, v):
            x.copy_(rand(g, *x.shape, dtype=torch.bfloat16))
        bias.table.copy_(rand(g, Hq, 20))
        c.dlens.copy_(torch.tensor([int(torch.randint(1, m + 1, (1,), generator=g)) for m in c.lens], dtype=torch.int32))
    fill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        fill()
        graph.replay()
        got = [x.clone() for x in (out, one)]
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], one)


def test_a_bias_that_hides_and_caps_far_below_the_scores():
    """Buckets hidden by -inf and by the lowest number; scores many times the cap."""
    g, Hq, Hk, d = gen(12), 6, 3, 72
    for dt in (torch.float32, torch.bfloat16):
        c = Paged(g, [300, 40, 0], 20, 16, Hk, d, dt)
        new = [3, 25, 2]
        last, pos = [], []
        for m, n in zip(c.lens, new):
            l, depth = tree_of(g, n, "tree")
            last += list(l)
            pos += [m + y for y in depth]
        last, pos = torch.tensor(last, dtype=torch.int32), torch.tensor(pos, dtype=torch.int32)
        x = {n: rand(g, 30, H, d, dtype=dt) * 3 for n, H in (("q", Hq), ("k", Hk), ("v", Hk))}
        table, bounds = rand(g, Hq, 6), torch.tensor([1, 2, 5, 20, 100], dtype=torch.int32)
        table[0, 1], table[2, :3], table[5] = -math.inf, torch.finfo(torch.float32).min, -math.inf
        items = hot.NewItems(offsets(new).to(DEV), 30, 25, last=last.to(DEV), positions=pos.to(DEV))
        out = run_tree(c, x, items, hot.RelBias(table.to(DEV), bounds.to(DEV)), None, 0.5, "rows")
        table = torch.where(table <= -60000.0, torch.full_like(table, -math.inf), table)
        check_tree(c, new, x, (pos, last, None, table, bounds, d ** -0.5, 0.5), out)
        assert not out[:, 5].any()
        q = x["q"][:3]
        ws = hot.alloc_cache_attn_bias_workspace(c.cache, Hq, 300)
        one = torch.full_like(q, NAN).to(DEV)
        hot.dlrm_cache_attn_bias(c.cache, c.dlens, 300, hot.RelBias(table.to(DEV), bounds.to(DEV)), q.to(DEV), one, ws, cap=0.5)
        for s, m in enumerate(c.lens):
            want, tol = ref.cached(q[s:s + 1], c.k[s], c.v[s], None, None, torch.tensor([m - 1]), None, None, table, bounds, d ** -0.5, 0.5)
            close(one[s:s + 1], want, tol, "sequence %d" % s)


def test_drafts_are_run_in_a_tree_and_a_path_of_them_is_kept():
    """Drafts of every user in one call; the items on the way to one of them are then stored, and that item alone, run over the cache, is what it was in the tree."""
    g, Hq, Hk, d, page = gen(21), 8, 4, 128, 32
    lens, new = [70, 1, 300], [24, 5, 17]
    c = Paged(g, lens, 12, page, Hk, d, torch.bfloat16)
    B, T, starts = 3, sum(new), offsets(new)
    pool = torch.full((2, 36, Hk, page, d), NAN, dtype=torch.bfloat16, device=DEV)
    cache = hot.KvCache(pool[0], pool[1], torch.randperm(36, generator=g).to(torch.int32).view(3, 12).to(DEV))
    bias = hot.RelBias(torch.randn(Hq, 40, device=DEV), hot.relative_bounds(40, 200, device=DEV))
    rope = lambda pos: hot.QkRope(pos.to(torch.int32).to(DEV), Hq, Hk, d, inv_freq=hot.rope_frequencies(d, device=DEV))

    def store(users, pos, q, k, v):
        hot.dlrm_qk_rope_append(rope(pos), q, k, v, torch.empty_like(q), cache, users.to(torch.int32).to(DEV))
    for s, n in enumerate(lens):
        store(torch.full((n,), s), torch.arange(n), rand(g, n, Hq, d, dtype=torch.bfloat16).to(DEV), c.k[s].to(DEV), c.v[s].to(DEV))
    parents = [[-1] + [int(torch.randint(-1, i, (1,), generator=g)) for i in range(1, n)] for n in new]
    order, last, depth = zip(*(hot.tree_order(p) for p in parents))
    pos = torch.tensor([m + y for m, x in zip(lens, depth) for y in x])
    q, k, v = (rand(g, T, H, d, dtype=torch.bfloat16).to(DEV) for H in (Hq, Hk, Hk))   # in depth-first order
    qr, kr, out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    hot.dlrm_qk_rope_fwd(rope(pos), q, k, qr, kr)
    items = hot.NewItems(starts.to(DEV), T, max(new), last=torch.tensor(sum(last, []), dtype=torch.int32, device=DEV), positions=pos.to(torch.int32).to(DEV))
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    hot.dlrm_cache_tree_attn(cache, dl, max(lens), items, qr, kr, v, out, hot.alloc_cache_tree_attn_workspace(cache, Hq, max(lens), items), bias=bias, cap=30.0)
    ends = [max(range(n), key=lambda i: x[i]) for n, x in zip(new, depth)]   # the deepest draft of each
    path = [[j for j in range(e + 1) if l[j] >= e] for e, l in zip(ends, last)]
    assert [len(x) for x in path] == [depth[s][ends[s]] + 1 for s in range(B)]
    rows = torch.tensor([int(starts[s]) + j for s in range(B) for j in path[s]])
    users = torch.tensor([s for s in range(B) for _ in path[s]])
    a = rows.to(DEV)
    store(users, pos[rows], q[a], k[a], v[a])
    now = [m + len(x) for m, x in zip(lens, path)]
    at = torch.tensor([int(starts[s]) + ends[s] for s in range(B)], device=DEV)
    one = torch.empty(B, Hq, d, dtype=torch.bfloat16, device=DEV)
    hot.dlrm_cache_attn_bias(cache, torch.tensor(now, dtype=torch.int32, device=DEV), max(now), bias, qr[at], one,
                             hot.alloc_cache_attn_bias_workspace(cache, Hq, max(now)), cap=30.0)
    # both round one number to bf16, and the tree's weights are rounded once more
    close(one, out[at].double().cpu(), (2 ** -7 * out[at].double().abs() + 2 ** -8 * 4.5).cpu(), "the kept draft")


def test_calls_on_two_streams_at_once_are_what_they_are_alone():
    """Each with a workspace of its own, on streams other than the tensors'."""
    g, Hq, Hk, d = gen(33), 8, 2, 128
    c = Paged(g, [9000, 40, 700], 150, 64, Hk, d, torch.bfloat16)
    new, T = [20, 1, 37], 58
    last = torch.tensor(sum((tree_of(g, m, "tree")[0] for m in new), []), dtype=torch.int32, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) + 9000
    items = hot.NewItems(offsets(new).to(DEV), T, 37, last=last, positions=pos)
    bias = hot.RelBias(torch.randn(Hq, 50, device=DEV), hot.relative_bounds(50, 3000, device=DEV))
    x = [[rand(g, T, H, d, dtype=torch.bfloat16).to(DEV) for H in (Hq, Hk, Hk)] for _ in range(2)]

    def step(i, out, one, ws, ws1):
        hot.dlrm_cache_tree_attn(c.cache, c.dlens, 9000, items, *x[i], out, ws, bias=bias)
        hot.dlrm_cache_attn_bias(c.cache, c.dlens, 9000, bias, x[i][0][:3], one, ws1)

    room = lambda: (torch.full((T, Hq, d), NAN, dtype=torch.bfloat16, device=DEV), torch.full((3, Hq, d), NAN, dtype=torch.bfloat16, device=DEV),
                    hot.alloc_cache_tree_attn_workspace(c.cache, Hq, 9000, items), hot.alloc_cache_attn_bias_workspace(c.cache, Hq, 9000))
    alone, both, streams = [room(), room()], [room(), room()], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(2):
        step(i, *alone[i])
    torch.cuda.synchronize()
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                step(i, *both[i])
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m", [3, 20, 70])
def test_infinite_values_that_are_seen_stay_infinite(dtype, m):
    """12, 80 and 280 columns: a weight's two parts both meet the value, and zero times an infinity would be NaN.  Other columns are what they are without it."""
    g, Hq, Hk, d, dt = gen(60 + m), 8, 2, 64, DT[dtype]
    c = Paged(g, [300, 40], 20, 16, Hk, d, dt)
    x = {n: rand(g, 2 * m, H, d, dtype=dt) for n, H in (("q", Hq), ("k", Hk), ("v", Hk))}
    items = hot.NewItems(offsets([m, m]).to(DEV), 2 * m, m)
    plain = run_tree(c, x, items, None, None, 0.0, "rows")
    page = c.cache.table[0, 1]
    c.dev[1][page.long(), :, 5, 7] = math.inf   # item 21 of the first sequence
    x["v"][0, :, 9] = -math.inf                 # its first new item, which all of them see
    out = run_tree(c, x, items, None, None, 0.0, "rows")
    assert (out[:m, :, 7] == math.inf).all() and (out[:m, :, 9] == -math.inf).all()
    rest = [i for i in range(d) if i not in (7, 9)]
    assert torch.equal(out[:, :, rest], plain[:, :, rest]) and torch.equal(out[m:], plain[m:])
