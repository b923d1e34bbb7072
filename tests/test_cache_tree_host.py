"""Attention of new items over a paged cache (dlrm_cache_attn_bias, dlrm_cache_tree_attn) without a GPU: refusals, workspaces, the order of a tree."""
import ctypes as C
import random

import pytest
import torch

import paper_1906_00091_amd as hot
from paper_1906_00091_amd import binding

from test_history_host import BAD_CACHE, BAD_HEADS, NULL, P, SHAPE, WORKSPACE, cache, heads
from test_relative_bias_host import BAD_BIAS, bias

SCORE = [(dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(cap=-1.0), SHAPE), (dict(cap=float("inf")), SHAPE)]


def items(**kw):
    a = dict(T=6, max_items=4, off=P, last=P, positions=P)
    a.update(kw)
    return binding._NewItemsC(**a)


def one(c=None, b=None, lens=P, max_len=64, Hq=4, slopes=None, scale=0.125, cap=0.0, ws=P, n=1 << 40, **kw):
    h = {"q": heads(), "o": heads()}
    h.update(kw)
    return hot.lib().dlrm_cache_attn_bias(c, lens, max_len, b, Hq, h["q"], h["o"], slopes, scale, cap, ws, n, None)


def tree(c=None, x=None, b=None, lens=P, max_len=64, Hq=4, slopes=None, scale=0.125, cap=0.0, ws=P, n=1 << 40, **kw):
    h = {m: heads() for m in ("q", "k", "v", "o")}
    h.update(kw)
    return hot.lib().dlrm_cache_tree_attn(c, lens, max_len, x, Hq, h["q"], h["k"], h["v"], h["o"], b, slopes, scale, cap, ws, n, None)


def test_refusals_of_one_new_item_with_a_bias():
    assert one(None, bias()) == NULL and one(cache(), None) == NULL and one(cache(), bias(), lens=None) == NULL
    for kw, want in BAD_CACHE:
        assert one(cache(**kw), bias()) == want, kw
    for kw, want in BAD_BIAS:
        assert one(cache(), bias(**kw)) == want, kw
    for kw, want in SCORE + [(dict(max_len=0), SHAPE), (dict(Hq=3), SHAPE), (dict(Hq=0), SHAPE)]:
        assert one(cache(), bias(), **kw) == want, kw
    for n in ("q", "o"):
        for kw, want in BAD_HEADS:
            assert one(cache(), bias(), **{n: heads(**kw)}) == want, (n, kw)


def test_refusals_of_new_items():
    assert tree(None, items()) == NULL and tree(cache(), None) == NULL and tree(cache(), items(), lens=None) == NULL
    for kw, want in BAD_CACHE:
        assert tree(cache(**kw), items()) == want, kw
    for kw, want in BAD_BIAS:
        assert tree(cache(), items(), bias(**kw)) == want, kw
    for kw, want in SCORE + [(dict(max_len=-1), SHAPE), (dict(Hq=3), SHAPE)]:
        assert tree(cache(), items(), **kw) == want, kw
    for kw, want in ((dict(T=-1), SHAPE), (dict(T=1 << 31), SHAPE), (dict(max_items=0), SHAPE), (dict(off=None), NULL),
                     (dict(T=2 ** 31 - 1, max_items=2 ** 31 - 1), SHAPE)):
        assert tree(cache(), items(**kw)) == want, kw
    for kw in (dict(slopes=P), dict(b=bias())):   # distances need places
        assert tree(cache(), items(positions=None), **kw) == NULL, kw
    for n in ("q", "k", "v", "o"):
        for kw, want in BAD_HEADS:
            assert tree(cache(), items(), **{n: heads(**kw)}) == want, (n, kw)
    # nothing to answer is no error, and nothing is launched
    assert tree(cache(), items(T=0, last=None, positions=None), b=bias(), ws=None, n=0, **{n: heads(data=None) for n in ("q", "k", "v", "o")}) == 0


def test_workspaces():
    L = hot.lib()
    long = cache(B=1, table_cols=1 << 14, n_pages=1 << 14)
    need = L.dlrm_cache_attn_bias_workspace_bytes(C.byref(long), 4, 1 << 17)
    assert need > 256
    for ws, n in ((None, need), (P + 128, need), (P, need - 1)):
        assert one(long, bias(), max_len=1 << 17, ws=ws, n=n) == WORKSPACE
    x = items(T=64, max_items=64)
    need = L.dlrm_cache_tree_attn_workspace_bytes(C.byref(long), C.byref(x), 4, 1 << 17)
    for ws, n in ((None, need), (P + 128, need), (P, need - 1)):
        assert tree(long, x, max_len=1 << 17, ws=ws, n=n) == WORKSPACE
    assert L.dlrm_cache_attn_bias_workspace_bytes(C.byref(cache(B=0)), 4, 64) == 0 and L.dlrm_cache_attn_bias_workspace_bytes(C.byref(cache()), 4, 0) == 0
    assert L.dlrm_cache_tree_attn_workspace_bytes(C.byref(cache()), None, 4, 64) == 0
    assert L.dlrm_cache_tree_attn_workspace_bytes(C.byref(cache()), C.byref(items(max_items=0)), 4, 64) == 0


def chunks(c, x, Hq, max_len):
    """Chunks of the length for a call, as the library cuts it: workgroups of 16, 32 or 64 columns, 1024 of them, chunks of 256 keys or more in
    steps of 128, no more pages than a table of 1024 holds."""
    n = max(1, min(x.max_items, x.T))
    cols = n * (Hq // c.Hk)
    tile = 16 if cols <= 16 else 32 if cols <= 32 or c.dtype == hot.F32 else 64
    groups = c.B * c.Hk * -(-cols // tile)
    total = min(max_len, c.table_cols * c.page) + n
    chunk = min(-(-max(256, -(-groups * total // 1024)) // 128) * 128, 1023 * c.page, total)
    return (total - 1) // chunk + 1


def test_the_workspace_for_a_bound_serves_every_smaller_one():
    rng = random.Random(5)
    for _ in range(300):
        Hk = rng.choice([1, 2, 4])
        Hq = Hk * rng.choice([1, 4, 8])
        c = cache(B=rng.choice([1, 3, 8, 100]), Hk=Hk, page=rng.choice([1, 8, 64]), table_cols=rng.choice([3, 200, 5000]), n_pages=9, d=rng.choice([8, 128]),
                  dtype=rng.choice([hot.F32, hot.BF16]))
        x = items(T=rng.choice([1, 7, 500]), max_items=rng.choice([1, 7, 64, 1000]))
        top = rng.choice([0, 1, 300, 8256, 100000])
        need = hot.lib().dlrm_cache_tree_attn_workspace_bytes(C.byref(c), C.byref(x), Hq, top)
        for max_len in {top, top // 2, top * 31 // 32, min(top, 256), 0}:
            n = chunks(c, x, Hq, max_len)
            assert n == 1 or n * x.T * Hq * (c.d + 2) * 4 <= need


def test_binding_refuses():
    off = torch.tensor([0, 2, 4])
    i32 = torch.zeros(4, dtype=torch.int32)
    for kw in (dict(last=i32[:3]), dict(last=i32.long()), dict(positions=i32[:2])):
        with pytest.raises(ValueError):
            hot.NewItems(off, 4, 2, **kw)
    with pytest.raises(ValueError):
        hot.NewItems(off.int(), 4, 2)
    pool = torch.zeros(2, 8, 2, 16, 8)
    c = hot.KvCache(pool[0], pool[1], torch.zeros(3, 2, dtype=torch.int32))
    q, k = torch.zeros(4, 4, 8), torch.zeros(4, 2, 8)
    with pytest.raises(ValueError, match="2 sequences for a cache of 3"):
        hot.dlrm_cache_tree_attn(c, torch.zeros(3, dtype=torch.int32), 32, hot.NewItems(off, 4, 2), q, k, k, q, None)
    with pytest.raises(ValueError, match="heads for 4"):
        hot.dlrm_cache_attn_bias(c, torch.zeros(3, dtype=torch.int32), 32, hot.RelBias(torch.zeros(2, 1), None), torch.zeros(3, 4, 8), torch.zeros(3, 4, 8), None)


def test_the_order_of_a_tree():
    order, last, depth = hot.tree_order([-1, 0, 0, 1, -1, 2, 1, 4])
    #   0 - 1 - 3
    #         - 6
    #     - 2 - 5
    #   4 - 7
    assert order == [0, 1, 3, 6, 2, 5, 4, 7] and depth == [0, 1, 2, 2, 1, 2, 0, 1] and last == [5, 3, 2, 3, 5, 5, 7, 7]
    assert hot.tree_order([]) == ([], [], []) and hot.tree_order([-1, -1]) == ([0, 1], [0, 1], [0, 0])
    n = 5000   # a chain far deeper than Python's own recursion
    assert hot.tree_order([i - 1 for i in range(n)]) == (list(range(n)), [n - 1] * n, list(range(n)))
    for bad in ([1, 0], [0], [-2], [3, -1]):
        with pytest.raises(ValueError):
            hot.tree_order(bad)


@pytest.mark.parametrize("seed", range(5))
def test_an_item_of_a_tree_sees_its_ancestors_and_itself(seed):
    rng = random.Random(seed)
    parents = [-1]
    for i in range(1, 60):
        parents.append(rng.randrange(-1, i))
    names = list(range(60))
    rng.shuffle(names)               # parents may come after their children
    mixed = [0] * 60
    for i, p in enumerate(parents):
        mixed[names[i]] = -1 if p < 0 else names[p]
    order, last, depth = hot.tree_order(mixed)
    at = {x: i for i, x in enumerate(order)}
    for i, x in enumerate(order):
        above, y = {i}, mixed[x]
        while y >= 0:
            above.add(at[y])
            y = mixed[y]
        assert above == {j for j in range(60) if j <= i <= last[j]} and depth[i] == len(above) - 1


def test_a_call_without_items_is_checked_like_any_other():
    none = dict(ws=None, n=0, **{n: heads(data=None) for n in ("q", "k", "v", "o")})
    x = items(T=0, last=None, positions=None)
    assert tree(cache(), x, **none) == 0
    for kw, want in SCORE:
        assert tree(cache(), x, **dict(none, **kw)) == want, kw
    for n in ("q", "k", "v", "o"):
        assert tree(cache(), x, **dict(none, **{n: heads(data=P + 8)})) == SHAPE, n
    assert tree(cache(), x, lens=None, **none) == NULL


@pytest.mark.parametrize("B,Hk", [(1 << 27, 16), ((1 << 28) - 1, 16), (1 << 28, 16), (2 ** 31 - 1, 1), (2 ** 31 - 1, 1024)])
@pytest.mark.parametrize("page", [1, 16])
def test_batches_whose_sequences_times_heads_pass_32_bits(B, Hk, page):
    """2^31 and more groups of a sequence and a key head: none is cut but where a chunk's table of 1024 pages ends."""
    c, max_len, d = cache(B=B, Hk=Hk, d=8, page=page, table_cols=1 << 16), 1 << 16, 8
    pieces = -(-max_len // (1023 * page))
    need = hot.lib().dlrm_cache_attn_bias_workspace_bytes(C.byref(c), Hk, max_len)
    assert need >= B * Hk * pieces * (d + 2) * 4
    x = items(T=2 ** 31 - 1, max_items=1)
    need = hot.lib().dlrm_cache_tree_attn_workspace_bytes(C.byref(c), C.byref(x), Hk, max_len)
    assert need >= x.T * Hk * -(-(max_len + 1) // (1023 * page)) * (d + 2) * 4
    x = items(T=2 ** 31 - 1, max_items=1 << 20)   # a loose bound: 2^16 and more blocks of columns for each sequence
    assert hot.lib().dlrm_cache_tree_attn_workspace_bytes(C.byref(c), C.byref(x), Hk, max_len) >= x.T * Hk * pieces * (d + 2) * 4
