"""Buckets of a learned bias at the ends of what a caller may give: the farthest distances that integers have, through the kernels for few and for many new
items, against the number of bounds that are at most each distance."""
import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from history_ref import close, offsets
from test_gpu_cache_tree import Paged, up
from test_gpu_relative_bias import DEV, DT, NAN, gen, rand

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
