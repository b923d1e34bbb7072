"""Workspace of the attention over the cache, without a GPU: what was allocated for the longest histories serves shorter ones."""
import ctypes as C
import random

import pytest

import paper_1906_00091_amd as hot
from paper_1906_00091_amd import binding


def need(B, Hq, Hk, d, page, max_len, cols=None):
    c = binding._KvCacheC(0x10000, 0x10000, 0x10000, B, (max_len + page - 1) // page if cols is None else cols, 1 << 20, page, Hk, d, hot.BF16)
    return hot.lib().dlrm_cache_attn_workspace_bytes(C.byref(c), Hq, max_len)


@pytest.mark.parametrize("B,Hq,Hk,d,page", [(64, 4, 4, 64, 16), (8, 16, 4, 128, 64), (1, 16, 4, 128, 64), (1, 40, 1, 64, 1), (3, 6, 3, 72, 8), (300, 8, 8, 32, 1024),
                                           (2048, 4, 4, 64, 16)])
def test_a_larger_bound_never_needs_less(B, Hq, Hk, d, page):
    rng, cols, last = random.Random(B), (1 << 30) // page, 0
    lengths = sorted([*range(1, 9000, 13), *(int(2 ** rng.uniform(13, 30)) for _ in range(3000)), 1 << 30])
    for n in lengths:
        b = need(B, Hq, Hk, d, page, n, cols)
        assert b >= last and b % 256 == 0, (n, b, last)
        last = b


@pytest.mark.parametrize("shape,lengths", [((64, 4, 4, 64, 16), (832, 1088)), ((8, 16, 4, 128, 64), (8000, 8256)), ((1, 16, 4, 128, 64), (65344, 65600))])
def test_lengths_whose_chunks_are_rounded_up(shape, lengths):
    """Pairs where the shorter bound is cut into more chunks than the longer one."""
    a, b = (need(*shape, n, cols=1 << 14) for n in lengths)
    assert b >= a


def test_a_sequence_of_too_many_workgroups_is_refused():
    """2^31 - 1 pages of one item and 16 key heads: 2^21 chunks times 16.  With 2 key heads the call is refused for its missing workspace alone."""
    class HeadsC(C.Structure):
        _fields_ = [("data", C.c_void_p), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]
    top = (1 << 31) - 1
    for Hk, status in ((16, -2), (2, -4)):
        c = binding._KvCacheC(0x10000, 0x10000, 0x10000, 1, top, 4, 1, Hk, 8, hot.BF16)
        x = C.byref(HeadsC(0x10000, Hk * 8, 8))
        assert hot.lib().dlrm_cache_attn(C.byref(c), 0x10000, top, Hk, x, x, None, 1.0, 0.0, None, 0, None) == status
