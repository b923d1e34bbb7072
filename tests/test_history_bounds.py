"""Bounds of the attention over sequences, without a GPU: how loose and how large they may be."""
import ctypes as C

import pytest

import paper_1906_00091_amd as hot
from paper_1906_00091_amd import binding

P = 0x10000
MOST = (1 << 31) - 1025


class HeadsC(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]


def workspace(Hq=4, Hk=2, **kw):
    a = dict(B=2, causal=1, Tq=8, Tk=8, max_q=4, max_k=4, q_off=P, k_off=P, prefix=None, slopes=None, scale=0.125, cap=0.0)
    a.update(kw)
    return hot.lib().dlrm_seq_attn_bwd_workspace_bytes(C.byref(binding._SeqBatchC(**a)), Hq, Hk, 64, hot.BF16)


@pytest.mark.parametrize("Tq,Tk", [(8, 8), (3, 9000), (5000, 1)])
def test_a_bound_above_the_total_counts_as_the_total(Tq, Tk):
    want = workspace(Tq=Tq, Tk=Tk, max_q=Tq, max_k=Tk)
    assert want > 0
    for q, k in ((Tq + 1, Tk), (Tq, Tk + 1), ((1 << 31) - 1, (1 << 31) - 1)):
        assert workspace(Tq=Tq, Tk=Tk, max_q=q, max_k=k) == want


def test_sequences_of_more_items_than_32_bits_count():
    """Refused as a shape before anything is launched: a tile past the end of a longer one would have no number."""
    x = C.byref(HeadsC(P, 1024, 64))
    for Hq, Hk, kw, fits in ((1, 1, dict(Tk=MOST, max_k=MOST), True), (1, 1, dict(Tk=MOST + 1, max_k=MOST + 1), False),
                             (1, 1, dict(Tq=MOST, max_q=MOST), True), (1, 1, dict(Tq=MOST + 1, max_q=MOST + 1), False),
                             (8, 1, dict(Tq=1 << 28, max_q=1 << 28), False), (8, 8, dict(Tq=1 << 28, max_q=1 << 28), True),
                             (8, 1, dict(Tq=1 << 28, max_q=1 << 27), True)):
        assert (workspace(Hq, Hk, **kw) > 0) == fits, (Hq, Hk, kw)
        if not fits:
            a = dict(B=2, causal=1, Tq=8, Tk=8, max_q=4, max_k=4, q_off=P, k_off=P, prefix=None, slopes=None, scale=0.125, cap=0.0)
            a.update(kw)
            s = C.byref(binding._SeqBatchC(**a))
            assert hot.lib().dlrm_seq_attn_fwd(s, Hq, Hk, 64, hot.BF16, x, x, x, x, P, None) == -2
            assert hot.lib().dlrm_seq_attn_bwd(s, Hq, Hk, 64, hot.BF16, x, x, x, x, P, x, x, x, x, P, 1 << 62, None) == -2
