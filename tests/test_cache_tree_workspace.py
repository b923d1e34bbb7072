"""Workspaces of new items and of biased attention over the cache, without a GPU: what was allocated for a bound on the length holds the chunks of every smaller one, by
the very rule that the library cuts with (tree_cut.h, built for the host)."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

import paper_1906_00091_amd as hot

from test_cache_tree_host import items
from test_history_host import cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    lib = str(tmp_path_factory.mktemp("cut") / "libtree_cut.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_1906_00091_amd", "csrc"),
                    os.path.join(ROOT, "tests", "tree_cut_driver.cpp"), "-o", lib], check=True)
    f, to = C.CDLL(lib).tree_cut, (C.c_int64 * 4)()

    def call(c, Hq, max_len, max_items):
        f(C.byref(c), Hq, max_len, max_items, to)
        return tuple(to)   # tiles, chunk, splits, blocks
    return call


def log(rng, top):
    return int(2 ** rng.uniform(0, top))


def test_the_workspace_for_a_bound_holds_the_chunks_of_every_smaller_one(cut):
    rng, seen, more, L = random.Random(11), set(), 0, hot.lib()
    for _ in range(6000):
        Hk, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8, 64, 65, 80])
        Hq, page = Hk * G, 2 ** rng.randint(0, 10)
        cols = max(1, min(log(rng, 18), (2 ** 31 - 1) // page))
        c = cache(B=log(rng, 13), Hk=Hk, page=page, table_cols=cols, n_pages=9, d=8, dtype=rng.choice([hot.F32, hot.F16, hot.BF16]))
        # around the columns that the cut changes at, and anywhere
        n = rng.choice([0, 1, 16 // G, 16 // G + 1, 32 // G, 32 // G + 1, 128 // G, 128 // G + 1, log(rng, 11), log(rng, 11)])
        top = max(1, min(log(rng, 24), 2 * cols * page))
        if n:
            x = items(T=rng.choice([n, 7 * n]), max_items=n)
            rows, need = x.T * Hq, L.dlrm_cache_tree_attn_workspace_bytes(C.byref(c), C.byref(x), Hq, top)
        else:
            rows, need = c.B * Hq, L.dlrm_cache_attn_bias_workspace_bytes(C.byref(c), Hq, top)
        most = cut(c, Hq, top, n)[2]
        for max_len in {top, top - 1, top // 2, top * 31 // 32, top * 7 // 8, log(rng, 24) % (top + 1), rng.randint(0, top), 1, 0 if n else 1}:
            tiles, chunk, splits, blocks = cut(c, Hq, max_len, n)
            total = min(max_len, cols * page) + n
            assert (splits - 1) * chunk < max(total, 1) <= splits * chunk or total == 0
            assert chunk <= 1023 * page and blocks * 16 * tiles >= n * G
            assert splits == 1 or splits * rows * (c.d + 2) * 4 <= need, (tiles, chunk, splits, top, max_len, n, G)
            seen.add((tiles, min(splits, 3)))
            more += splits > most
    assert seen == {(t, s) for t in (1, 2, 8, 16) for s in (1, 2, 3)} and more > 50   # (shorter bounds that are cut into more chunks are among them)


@pytest.mark.parametrize("B,Hk,items_", [(2 ** 31 - 1, 1024, 1), (2 ** 31 - 1, 1, 2 ** 31 - 2 ** 20), (1 << 28, 16, 0), (1, 1, 2 ** 31 - 2 ** 20)])
def test_the_largest_calls_are_counted_without_overflow(cut, B, Hk, items_):
    """(the driver is built with the undefined-behaviour sanitizer, which ends the process)"""
    c = cache(B=B, Hk=Hk, page=1, table_cols=2 ** 20 - 2048, n_pages=9, d=8)
    tiles, chunk, splits, blocks = cut(c, Hk, 2 ** 31 - 1, items_)
    assert 1 <= chunk <= 1023 and splits == -(-(2 ** 20 - 2048 + items_) // chunk) and blocks == -(-max(1, items_) // (16 * tiles))
