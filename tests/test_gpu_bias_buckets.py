"""Buckets of a learned bias at the ends of what a caller may give: the farthest distances that integers have, through the kernels for few and for many new
items, and bounds that are there several times, against the number of bounds that are at most each distance."""
import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from history_ref import close, offsets
from test_gpu_cache_tree import Paged, up
from test_gpu_relative_bias import DEV, DT, NAN, gen, rand, run

pytestmark = pytest.mark.gpu
TOP = 2 ** 31 - 1

# places of a sequence's new items: all near the largest integer (a tile's distances fit one window), and some there and some at the other end
NEAR_TOP = [TOP, TOP - 1, TOP - 31, TOP, TOP - 7]
APART = [TOP, 0, TOP - 1, 5, TOP - 40]
FARTHEST = [
    # type, query heads, key heads, d, cached, new items, places, bounds
    ("f32", 2, 1, 16, [3, 40], 5, NEAR_TOP, [1, 2, 3, 5]),                       # n = 5, searched as if there were 8
    ("f32", 2, 1, 16, [3, 40], 5, NEAR_TOP, [3, TOP]),                           # the last bound is in reach
    ("f32", 3, 1, 32, [40, 0], 5, APART, [-2 ** 31, -7, 0, TOP]),
    ("bf16", 2, 2, 64, [70, 1], 5, APART, [-TOP, TOP - 60, TOP - 35, TOP - 1, TOP]),
    ("bf16", 4, 1, 64, [70, 33], 11, NEAR_TOP, [-2 ** 31, TOP - 40]),            # 44 columns: the kernel for many
    ("bf16", 4, 1, 64, [70, 33], 11, APART, [-2 ** 31, -7, 0, TOP]),
    ("f32", 8, 1, 72, [130, 0], 9, APART, [1, 2, 3, 5]),
    ("f16", 8, 1, 128, [130, 64], 40, NEAR_TOP, [TOP - 130 + i for i in range(100)]),
    ("f16", 8, 1, 128, [130, 64], 40, APART, [i - 16 for i in range(32)]),       # n = 33, searched as if there were 64
]


@pytest.mark.parametrize("i", range(len(FARTHEST)))
def test_the_farthest_distances_have_their_own_buckets(i):
    dt, Hq, Hk, d, lens, m, places, bounds = FARTHEST[i]
    print("[case]", i, FARTHEST[i], flush=True)
    g, dt, B, n = gen(70 + i), DT[dt], len(lens), len(bounds) + 1
    c = Paged(g, lens, max(1, -(-max(lens) // 16)), 16, Hk, d, dt)
    x = {name: rand(g, B * m, H, d, dtype=dt) for name, H in (("q", Hq), ("k", Hk), ("v", Hk))}
    pos = torch.tensor([places[j % len(places)] for j in range(m)] * B, dtype=torch.int64).to(torch.int32)
    last = torch.tensor([m - 1] * (B * m), dtype=torch.int32)
    table, bounds = rand(g, Hq, n), torch.tensor(bounds, dtype=torch.int64).to(torch.int32)
    items = hot.NewItems(offsets([m] * B).to(DEV), B * m, m, last=last.to(DEV), positions=pos.to(DEV))
    out = torch.full_like(x["q"], NAN).to(DEV)
    hot.dlrm_cache_tree_attn(c.cache, c.dlens, max(lens), items, *(x[name].to(DEV) for name in "qkv"), out,
                             hot.alloc_cache_tree_attn_workspace(c.cache, Hq, max(lens), items), bias=hot.RelBias(table.to(DEV), up(bounds)))
    for s in range(B):
        I = slice(s * m, (s + 1) * m)
        want, tol = ref.cached(x["q"][I], c.k[s], c.v[s], x["k"][I], x["v"][I], pos[I], last[I], None, table, bounds, d ** -0.5, 0.0)
        close(out[I], want, tol, "sequence %d" % s)


AGAIN = [
    [1, 2, 2, 3, 3, 3, 10, 40, 40, 300],
    [5] * 7,
    [40, 40],                                                   # a tile has one of these places, or none
    [-3, -3, 0, 0, 0, 7],
    [round(1.06 ** i) for i in range(100)],                     # as a logarithm is rounded
    [i // 2 for i in range(20, 147)],                           # 127 of them: 63 and 64 are not the same, ...
    [(i + 1) // 2 for i in range(20, 147)],                     # ... and here they are
    [8] * 60 + [9] * 10 + [100] * 57,
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(AGAIN)))
def test_bounds_that_are_there_several_times(i, dtype):
    """A bound counts as often as it is there, in every kernel: over sequences with the table's gradient, for one new item, for few and for many."""
    print("[case]", i, dtype, flush=True)
    g, dt, bounds = gen(90 + i), DT[dtype], torch.tensor(AGAIN[i], dtype=torch.int32)
    assert bool((bounds[1:] == bounds[:-1]).any()) and bool((bounds[1:] >= bounds[:-1]).all())
    Hq, Hk, d, n, lens = 4, 2, 32, len(AGAIN[i]) + 1, [130, 3, 400]
    table = rand(g, Hq, n)
    bias = hot.RelBias(table.to(DEV), bounds.to(DEV))
    off, T = offsets(lens), sum(lens)
    x = {name: rand(g, T, H, d, dtype=dt) for name, H in (("q", Hq), ("k", Hk), ("v", Hk), ("do", Hq))}
    causal = i % 2 == 0
    got = run(x, hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 400, 400, causal=causal), bias, "rows")
    want = ref.attention(x["q"], x["k"], x["v"], off, off, causal, None, None, table, bounds, d ** -0.5, 0.0, x["do"])
    for name in got:
        close(got[name], want[name], want[name + "_tol"], name)
    empty = torch.bincount(torch.cat([ref.buckets(torch.arange(1 - m if not causal else 0, m), bounds) for m in lens]), minlength=n) == 0
    assert empty.any() and not got["dtable"][:, empty.to(DEV)].any()
    c = Paged(g, lens, 30, 16, Hk, d, dt)
    q = rand(g, 3, Hq, d, dtype=dt)
    one = torch.full_like(q, NAN).to(DEV)
    hot.dlrm_cache_attn_bias(c.cache, c.dlens, 400, bias, q.to(DEV), one, hot.alloc_cache_attn_bias_workspace(c.cache, Hq, 400))
    for s, m in enumerate(lens):
        w, tol = ref.cached(q[s:s + 1], c.k[s], c.v[s], None, None, torch.tensor([m - 1]), None, None, table, bounds, d ** -0.5, 0.0)
        close(one[s:s + 1], w, tol, "one, sequence %d" % s)
    for m in (6, 40):   # 12 and 80 columns
        x = {name: rand(g, 3 * m, H, d, dtype=dt) for name, H in (("q", Hq), ("k", Hk), ("v", Hk))}
        pos, last = torch.cat([torch.arange(y, y + m) for y in lens]).to(torch.int32), torch.full((3 * m,), m - 1, dtype=torch.int32)
        items = hot.NewItems(offsets([m] * 3).to(DEV), 3 * m, m, positions=pos.to(DEV))
        out = torch.full_like(x["q"], NAN).to(DEV)
        hot.dlrm_cache_tree_attn(c.cache, c.dlens, 400, items, *(x[name].to(DEV) for name in "qkv"), out,
                                 hot.alloc_cache_tree_attn_workspace(c.cache, Hq, 400, items), bias=bias)
        for s in range(3):
            I = slice(s * m, (s + 1) * m)
            w, tol = ref.cached(x["q"][I], c.k[s], c.v[s], x["k"][I], x["v"][I], pos[I], last[I], None, table, bounds, d ** -0.5, 0.0)
            close(out[I], w, tol, "%d items, sequence %d" % (m, s))
