"""Operators that read a history in order, without a GPU: what the library refuses before it launches anything, what the binding
refuses, the frequencies, and the tests' own 64-bit forms against differences."""
import ctypes as C

import pytest
import torch

import paper_1906_00091_amd as hot
from paper_1906_00091_amd import binding

import history_ref as ref

P = 0x10000
NULL, SHAPE, DTYPE, WORKSPACE = -1, -2, -3, -4


class HeadsC(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_t", C.c_int64), ("stride_h", C.c_int64)]


def heads(data=P, st=1024, sh=64):
    return C.byref(HeadsC(data, st, sh))


def rope(**kw):
    a = dict(T=4, Hq=4, Hk=2, d=64, dtype=hot.BF16, rot=32, layout=0, positions=P, inv_freq=P, wq=P, wk=P, eps=1e-6, mscale=1.0)
    a.update(kw)
    return binding._QkRopeC(**a)


def seq(**kw):
    a = dict(B=2, causal=1, Tq=8, Tk=8, max_q=4, max_k=4, q_off=P, k_off=P, prefix=None, slopes=None, scale=0.125, cap=0.0)
    a.update(kw)
    return binding._SeqBatchC(**a)


def cache(**kw):
    a = dict(k=P, v=P, table=P, B=2, table_cols=4, n_pages=8, page=16, Hk=2, d=64, dtype=hot.BF16)
    a.update(kw)
    return binding._KvCacheC(**a)


BAD_HEADS = [(dict(data=None), NULL), (dict(data=P + 8), SHAPE), (dict(st=1020), SHAPE), (dict(st=32), SHAPE), (dict(sh=56), SHAPE),
             (dict(sh=68), SHAPE), (dict(st=-1024), SHAPE), (dict(st=1 << 24), SHAPE)]
BAD_ROPE = [(dict(dtype=3), DTYPE), (dict(Hq=0), SHAPE), (dict(Hk=-1), SHAPE), (dict(d=60), SHAPE), (dict(d=136), SHAPE), (dict(d=0), SHAPE),
            (dict(T=-1), SHAPE), (dict(T=1 << 31), SHAPE), (dict(rot=33), SHAPE), (dict(rot=66), SHAPE), (dict(rot=-2), SHAPE), (dict(layout=2), SHAPE),
            (dict(positions=None), NULL), (dict(inv_freq=None), NULL), (dict(eps=0.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(wq=P + 4), SHAPE),
            (dict(wk=P + 8), SHAPE)]
BAD_SEQ = [(dict(B=0), SHAPE), (dict(Tq=-1), SHAPE), (dict(Tk=1 << 31), SHAPE), (dict(max_q=-1), SHAPE), (dict(max_k=0), SHAPE), (dict(q_off=None), NULL),
           (dict(k_off=None), NULL), (dict(causal=2), SHAPE), (dict(causal=0, prefix=P), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE),
           (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(cap=-1.0), SHAPE), (dict(cap=float("inf")), SHAPE)]
BAD_SHAPE = [((4, 2, 64, 5), DTYPE), ((4, 3, 64, 2), SHAPE), ((0, 1, 64, 2), SHAPE), ((4, 0, 64, 2), SHAPE), ((4, 2, 20, 2), SHAPE), ((4, 2, 256, 2), SHAPE),
             ((2048, 2, 64, 2), SHAPE)]
BAD_CACHE = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(B=0), SHAPE), (dict(table_cols=0), SHAPE), (dict(n_pages=0), SHAPE),
             (dict(page=0), SHAPE), (dict(page=24), SHAPE), (dict(page=2048), SHAPE), (dict(k=P + 8), SHAPE), (dict(table_cols=1 << 28), SHAPE)]


def rope_fwd(r=None, **kw):
    h = {n: heads() for n in ("q", "k", "qo", "ko")}
    h.update(kw)
    return hot.lib().dlrm_qk_rope_fwd(r, h["q"], h["k"], h["qo"], h["ko"], None)


def rope_bwd(r=None, dwq=P, dwk=P, ws=P, n=1 << 30, **kw):
    h = {n: heads() for n in ("q", "k", "dqo", "dko", "dq", "dk")}
    h.update(kw)
    return hot.lib().dlrm_qk_rope_bwd(r, h["q"], h["k"], h["dqo"], h["dko"], h["dq"], h["dk"], dwq, dwk, ws, n, None)


def rope_append(r=None, c=None, seqs=P, **kw):
    h = {n: heads() for n in ("q", "k", "v", "qo")}
    h.update(kw)
    return hot.lib().dlrm_qk_rope_append(r, h["q"], h["k"], h["v"], h["qo"], c, seqs, None)


def seq_fwd(s=None, shape=(4, 2, 64, hot.BF16), lse=P, **kw):
    h = {n: heads() for n in ("q", "k", "v", "o")}
    h.update(kw)
    return hot.lib().dlrm_seq_attn_fwd(s, *shape, h["q"], h["k"], h["v"], h["o"], lse, None)


def seq_bwd(s=None, shape=(4, 2, 64, hot.BF16), lse=P, ws=P, n=1 << 30, **kw):
    h = {n: heads() for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    h.update(kw)
    return hot.lib().dlrm_seq_attn_bwd(s, *shape, h["q"], h["k"], h["v"], h["o"], lse, h["do"], h["dq"], h["dk"], h["dv"], ws, n, None)


def cache_attn(c=None, lens=P, max_len=64, Hq=4, scale=0.125, cap=0.0, ws=P, n=1 << 30, **kw):
    h = {n: heads() for n in ("q", "o")}
    h.update(kw)
    return hot.lib().dlrm_cache_attn(c, lens, max_len, Hq, h["q"], h["o"], None, scale, cap, ws, n, None)


def test_rotation_refuses_bad_arguments():
    for bad, status in BAD_ROPE:
        r = C.byref(rope(**bad))
        assert rope_fwd(r) == status and rope_bwd(r) == status and rope_append(r, C.byref(cache())) == status, bad
        assert hot.lib().dlrm_qk_rope_bwd_workspace_bytes(r) == 0, bad
    assert rope_fwd() == NULL and rope_bwd() == NULL and rope_append(None, C.byref(cache())) == NULL
    for bad, status in BAD_HEADS:
        for n in ("q", "k", "qo", "ko"):
            assert rope_fwd(C.byref(rope()), **{n: heads(**bad)}) == status, (n, bad)
        for n in ("q", "k", "dqo", "dko", "dq", "dk"):
            assert rope_bwd(C.byref(rope()), **{n: heads(**bad)}) == status, (n, bad)
    assert rope_fwd(C.byref(rope()), k=None) == NULL
    assert rope_bwd(C.byref(rope()), dwq=None) == NULL and rope_bwd(C.byref(rope()), dwk=None) == NULL
    need = hot.lib().dlrm_qk_rope_bwd_workspace_bytes(C.byref(rope()))
    assert need > 0 and need % 256 == 0
    assert rope_bwd(C.byref(rope()), ws=None) == WORKSPACE and rope_bwd(C.byref(rope()), n=need - 1) == WORKSPACE
    assert rope_bwd(C.byref(rope()), ws=P + 16) == WORKSPACE


def test_append_refuses_bad_arguments():
    for bad, status in BAD_CACHE:
        assert rope_append(C.byref(rope()), C.byref(cache(**bad))) == status, bad
    assert rope_append(C.byref(rope()), None) == NULL and rope_append(C.byref(rope()), C.byref(cache()), seqs=None) == NULL
    assert rope_append(C.byref(rope(rot=0, positions=None)), C.byref(cache())) == NULL
    assert rope_append(C.byref(rope(Hk=4)), C.byref(cache())) == SHAPE and rope_append(C.byref(rope(d=32)), C.byref(cache())) == SHAPE
    assert rope_append(C.byref(rope()), C.byref(cache(dtype=hot.F16))) == DTYPE
    for n in ("q", "k", "v", "qo"):
        assert rope_append(C.byref(rope()), C.byref(cache()), **{n: heads(data=P + 2)}) == SHAPE


def test_sequence_attention_refuses_bad_arguments():
    for bad, status in BAD_SEQ:
        s = C.byref(seq(**bad))
        assert seq_fwd(s) == status and seq_bwd(s) == status, bad
        assert hot.lib().dlrm_seq_attn_bwd_workspace_bytes(s, 4, 2, 64, hot.BF16) == 0
    for shape, status in BAD_SHAPE:
        assert seq_fwd(C.byref(seq()), shape) == status and seq_bwd(C.byref(seq()), shape) == status, shape
    for bad, status in BAD_HEADS:
        for n in ("q", "k", "v", "o"):
            assert seq_fwd(C.byref(seq()), **{n: heads(**bad)}) == status, (n, bad)
        for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
            assert seq_bwd(C.byref(seq()), **{n: heads(**bad)}) == status, (n, bad)
    assert seq_fwd() == NULL and seq_bwd() == NULL and seq_bwd(C.byref(seq()), lse=None) == NULL
    need = hot.lib().dlrm_seq_attn_bwd_workspace_bytes(C.byref(seq()), 4, 2, 64, hot.BF16)
    assert need > 0 and need % 256 == 0
    assert seq_bwd(C.byref(seq()), ws=None) == WORKSPACE and seq_bwd(C.byref(seq()), n=need - 1) == WORKSPACE
    assert seq_bwd(C.byref(seq()), ws=P + 128) == WORKSPACE


def test_cache_attention_refuses_bad_arguments():
    for bad, status in BAD_CACHE:
        assert cache_attn(C.byref(cache(**bad))) == status, bad
        assert hot.lib().dlrm_cache_attn_workspace_bytes(C.byref(cache(**bad)), 4, 64) == 0
    assert cache_attn() == NULL and cache_attn(C.byref(cache()), lens=None) == NULL
    for kw in (dict(max_len=0), dict(Hq=3), dict(Hq=0), dict(scale=0.0), dict(scale=float("nan")), dict(cap=-2.0)):
        assert cache_attn(C.byref(cache()), **kw) == SHAPE, kw
    assert cache_attn(C.byref(cache(dtype=9))) == DTYPE and cache_attn(C.byref(cache(d=12))) == SHAPE
    for bad, status in BAD_HEADS:
        for n in ("q", "o"):
            assert cache_attn(C.byref(cache()), **{n: heads(**bad)}) == status, (n, bad)
    long = C.byref(cache(B=1, table_cols=4096, page=64, n_pages=4096))
    need = hot.lib().dlrm_cache_attn_workspace_bytes(long, 4, 200000)
    assert need > 0 and need % 256 == 0
    assert cache_attn(long, max_len=200000, ws=None) == WORKSPACE and cache_attn(long, max_len=200000, n=need - 1) == WORKSPACE


def test_the_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(4, 2, 16)
    off = torch.tensor([0, 4])
    s = hot.SeqBatch(off, off, 4, 4, 4, 4)
    for bad in (torch.zeros(4, 16), torch.zeros(4, 16, 2).transpose(1, 2)):
        with pytest.raises(ValueError):
            hot.dlrm_seq_attn_fwd(s, bad, x, x, x.clone())
    with pytest.raises(hot.DlrmError):
        hot.dlrm_seq_attn_fwd(s, x.double(), x, x, x.clone())
    with pytest.raises(ValueError):
        hot.dlrm_seq_attn_fwd(s, x, x, x, torch.zeros(4, 1, 16))
    with pytest.raises(hot.DlrmError):
        hot.dlrm_seq_attn_fwd(s, x, x, x.half(), x)
    with pytest.raises(ValueError):
        hot.dlrm_seq_attn_fwd(s, x, x, x, x.clone(), lse=torch.zeros(7))
    with pytest.raises(ValueError):
        hot.SeqBatch(off.int(), off, 4, 4, 4, 4)
    with pytest.raises(ValueError):
        hot.dlrm_seq_attn_fwd(hot.SeqBatch(off, off, 4, 4, 4, 4, slopes=torch.zeros(3)), x, x, x, x.clone())
    with pytest.raises(ValueError):
        hot.KvCache(torch.zeros(2, 1, 8, 16), torch.zeros(2, 1, 8, 8), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError):
        hot.KvCache(torch.zeros(2, 1, 8, 16), torch.zeros(2, 1, 8, 16), torch.zeros(1, 2))
    with pytest.raises(ValueError):
        hot.QkRope(torch.zeros(4), 2, 2, 16)
    with pytest.raises(ValueError):
        hot.QkRope(None, 2, 2, 16)


def test_frequencies_stretched_evenly_and_by_parts():
    f = hot.rope_frequencies(64)
    assert f.dtype == torch.float32 and f.shape == (32,) and float(f[0]) == 1.0
    assert torch.allclose(hot.rope_frequencies(64, stretch=4.0), f / 4)
    p = hot.rope_frequencies(64, stretch=4.0, keep_turns=32.0, drop_turns=1.0, trained_length=2048)
    turns = 2048 * f / (2 * torch.pi)
    assert torch.equal(p[turns >= 32], f[turns >= 32]) and torch.allclose(p[turns <= 1], f[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and ((p[mid] < f[mid]) & (p[mid] > f[mid] / 4)).all()
    with pytest.raises(ValueError):
        hot.rope_frequencies(64, keep_turns=1.0)


def _difference(f, x, g, seed):
    """Central difference of <f(x), g> along a random step, and the step."""
    step = torch.randn(x.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
    e = 1e-5
    return float(((f(x + e * step) - f(x - e * step)) * g).sum() / (2 * e)), step


def test_reference_gradients_of_attention_against_differences():
    t = torch.Generator().manual_seed(2)
    d, Hq, Hk = 6, 4, 2
    qo, ko = ref.offsets([3, 5, 2]), ref.offsets([4, 5, 0])
    ref.UNIT[torch.float64], ref.TINY[torch.float64] = 2.0 ** -53, 0.0
    x = [torch.randn(n, H, d, generator=t, dtype=torch.float64) for n, H in ((10, Hq), (9, Hk), (9, Hk))]
    do = torch.randn(10, Hq, d, generator=t, dtype=torch.float64)
    pre, sl = torch.tensor([2, 0, 1]), torch.tensor([0.5, 0.25, 0.1, 0.0])
    how = (qo, ko, True, pre, sl, 0.4, 2.0)
    r = ref.attention(*x, *how, do)
    for i, n in enumerate(("dq", "dk", "dv")):
        f = lambda y: ref.attention(*(y if i == j else z for j, z in enumerate(x)), *how)["out"]
        slope, step = _difference(f, x[i], do, i)
        assert abs(slope - float((r[n] * step).sum())) < 1e-6 * (1 + abs(slope)), n


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_reference_gradients_of_the_rotation_against_differences(layout):
    t = torch.Generator().manual_seed(4)
    x, g = (torch.randn(5, 2, 16, generator=t, dtype=torch.float64) for _ in range(2))
    w = 1 + 0.1 * torch.randn(16, generator=t, dtype=torch.float64)
    how = (torch.arange(5), hot.rope_frequencies(12), 12, layout, 1e-3, 1.5)
    dx, dw = ref.rope_grad(x, w, g, *how)
    for i, (y, grad) in enumerate(((x, dx), (w, dw))):
        f = (lambda z: ref.rope(z, w, *how)) if i == 0 else (lambda z: ref.rope(x, z, *how))
        slope, step = _difference(f, y, g, i)
        assert abs(slope - float((grad * step).sum())) < 1e-6 * (1 + abs(slope))
