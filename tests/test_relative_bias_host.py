"""The learned relative position bias without a GPU: what the library and the binding refuse, the bounds, the workspaces, and the tests' own 64-bit form
against differences."""
import ctypes as C

import pytest
import torch

import paper_1906_00091_amd as hot
from paper_1906_00091_amd import binding

import bias_ref as ref
from history_ref import offsets
from test_history_host import BAD_HEADS, BAD_SEQ, BAD_SHAPE, DTYPE, NULL, P, SHAPE, WORKSPACE, heads, seq  # noqa: F401


def bias(**kw):
    a = dict(table=P, bounds=P, n=32)
    a.update(kw)
    return binding._RelBiasC(**a)


BAD_BIAS = [(dict(table=None), NULL), (dict(bounds=None), NULL), (dict(n=0), SHAPE), (dict(n=-1), SHAPE), (dict(n=129), SHAPE)]


def fwd(s=None, b=None, shape=(4, 2, 64, hot.BF16), lse=P, **kw):
    h = {n: heads() for n in ("q", "k", "v", "o")}
    h.update(kw)
    return hot.lib().dlrm_seq_attn_bias_fwd(s, b, *shape, h["q"], h["k"], h["v"], h["o"], lse, None)


def bwd(s=None, b=None, shape=(4, 2, 64, hot.BF16), lse=P, dtable=P, ws=P, n=1 << 40, **kw):
    h = {n_: heads() for n_ in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    h.update(kw)
    return hot.lib().dlrm_seq_attn_bias_bwd(s, b, *shape, h["q"], h["k"], h["v"], h["o"], lse, h["do"], h["dq"], h["dk"], h["dv"], dtable, ws, n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_refusals(call):
    assert call(None, bias()) == NULL and call(seq(), None) == NULL
    for kw, want in BAD_SEQ:
        assert call(seq(**kw), bias()) == want, kw
    for kw, want in BAD_BIAS:
        assert call(seq(), bias(**kw)) == want, kw
    for shape, want in BAD_SHAPE:
        assert call(seq(), bias(), shape) == want, shape
    for n in ("q", "k", "v", "o"):
        for kw, want in BAD_HEADS:
            assert call(seq(), bias(), **{n: heads(**kw)}) == want, (n, kw)
    # 32 items of one head to a wavefront: the last ones of each head may be empty, and rows are counted in 32 bits
    assert call(seq(Tq=2 ** 31 - 1, max_q=2 ** 30, Tk=1), bias()) == SHAPE


@pytest.mark.parametrize("call", [fwd, bwd])
def test_scales_whose_inverse_leaves_fp32(call):
    """Without a cap the scores' products start from the bias by the scale: 1 / scale and a bias of 60000 times it have to be numbers."""
    for scale in (2.0 ** -149, 2.0 ** -129, 2.0 ** -65, 2.0 ** 65, 2.0 ** 127):
        assert call(seq(scale=scale), bias()) == SHAPE, scale
        assert call(seq(scale=scale, cap=5.0), bias()) == SHAPE, scale
    assert hot.lib().dlrm_seq_attn_bias_bwd_workspace_bytes(C.byref(seq(scale=2.0 ** -129)), C.byref(bias()), 4, 2, 64, hot.BF16) == 0


def test_refusals_of_the_backward():
    for n in ("do", "dq", "dk", "dv"):
        for kw, want in BAD_HEADS:
            assert bwd(seq(), bias(), **{n: heads(**kw)}) == want, (n, kw)
    assert bwd(seq(), bias(), lse=None) == NULL and bwd(seq(), bias(), dtable=None) == NULL
    need = hot.lib().dlrm_seq_attn_bias_bwd_workspace_bytes(C.byref(seq()), C.byref(bias()), 4, 2, 64, hot.BF16)
    assert need >= 256
    for ws, n in ((None, need), (P + 128, need), (P, need - 1)):
        assert bwd(seq(), bias(), ws=ws, n=n) == WORKSPACE


def test_workspace_of_unsupported_shapes_is_none():
    need = hot.lib().dlrm_seq_attn_bias_bwd_workspace_bytes
    assert need(C.byref(seq(B=0)), C.byref(bias()), 4, 2, 64, hot.BF16) == 0
    assert need(C.byref(seq()), C.byref(bias(n=0)), 4, 2, 64, hot.BF16) == 0
    assert need(C.byref(seq()), None, 4, 2, 64, hot.BF16) == 0
    assert need(C.byref(seq()), C.byref(bias()), 4, 3, 64, hot.BF16) == 0
    # what is kept grows with the buckets, and holds at least the unbiased backward's
    s = seq(B=2048, Tq=200000, Tk=200000, max_q=200, max_k=200)
    sizes = [need(C.byref(s), C.byref(bias(n=n)), 4, 4, 64, hot.BF16) for n in (1, 32, 128)]
    assert sizes[0] < sizes[1] < sizes[2] and sizes[0] >= hot.lib().dlrm_seq_attn_bwd_workspace_bytes(C.byref(s), 4, 4, 64, hot.BF16)


def test_binding_refuses():
    t = torch.zeros(4, 8)
    b = torch.arange(1, 8, dtype=torch.int32)
    for table, bounds in ((t.double(), b), (t[:, ::2], b[:3]), (t[0], b), (t, b.long()), (t, b[:6]), (t, None)):
        with pytest.raises(ValueError):
            hot.RelBias(table, bounds)
    assert hot.RelBias(t[:, :1].contiguous(), None).n == 1
    off = torch.tensor([0, 4])
    s = hot.SeqBatch(off, off, 4, 4, 4, 4)
    x, x2 = torch.zeros(4, 4, 8), torch.zeros(4, 2, 8)
    with pytest.raises(ValueError, match="4 heads for 2"):
        hot.dlrm_seq_attn_bias_fwd(s, hot.RelBias(t, b), x2, x2, x2, x2)
    with pytest.raises(ValueError):
        hot.dlrm_seq_attn_bias_bwd(s, hot.RelBias(t, b), x, x, x, x, torch.zeros(4, 4), x, x, x, x, torch.zeros(4, 7), None)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("n,far", [(1, 5), (2, 1), (3, 100), (8, 16), (32, 128), (33, 300), (64, 2048), (128, 10), (128, 100000)])
def test_bounds(n, far, both):
    b = hot.relative_bounds(n, far, both).tolist()
    assert len(b) == n - 1 and all(x < y for x, y in zip(b, b[1:]))
    up = [x for x in b if x > 0]
    assert up[:1] == [1] * bool(up)
    if not both:
        assert up == b
    else:  # a distance of -x has a bucket of its own where x has
        down = [1 - x for x in b if x <= 0]
        assert len(down) == (n - 1) // 2 and len(up) == n - 1 - len(down)
        near = (len(down) + 1) // 2
        assert sorted(down)[:near] == up[:near] or len(up) != len(down)
    if len(up) >= 4 and far > 4 * len(up):
        assert up[-1] in (far, far + 1)


@pytest.mark.parametrize("causal,slopes,cap", [(True, False, 0.0), (False, True, 0.0), (True, True, 2.0)])
def test_the_64_bit_form_against_differences(causal, slopes, cap):
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    lens, klens, Hq, Hk, d = [3, 0, 6], [5, 2, 4], 4, 2, 8
    qo, ko = offsets(lens), offsets(klens)
    x = {"q": rand(9, Hq, d), "k": rand(11, Hk, d), "v": rand(11, Hk, d), "table": rand(Hq, 5)}
    bounds, do = torch.tensor([-2, 0, 1, 3]), rand(9, Hq, d)
    sl = rand(Hq).abs() if slopes else None
    pre = torch.tensor([2, 1, 3]) if causal else None
    ref.UNIT.setdefault(torch.float64, 2.0 ** -53)
    ref.TINY.setdefault(torch.float64, 0.0)

    def run(y, dout=None):
        return ref.attention(y["q"], y["k"], y["v"], qo, ko, causal, pre, sl, y["table"], bounds, 0.3, cap, dout)
    got = run(x, do)
    for n in x:
        grad = got["d" + n]
        for at in range(0, x[n].numel(), 7):
            sides = []
            for step in (1e-5, -1e-5):
                y = {m: t.clone() for m, t in x.items()}
                y[n].view(-1)[at] += step
                sides.append(float((run(y)["out"] * do).sum()))
            assert abs((sides[0] - sides[1]) / 2e-5 - float(grad.view(-1)[at])) < 1e-8, (n, at)


def test_plans_and_calls_refuse_arrays_on_several_devices():
    """(the other device is torch's own "meta" here: with a GPU it is the host, whose addresses a kernel must not get)"""
    meta = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="meta")
    table, bounds, off, i32 = torch.zeros(4, 8), hot.relative_bounds(8, 20), torch.tensor([0, 4]), torch.zeros(4, dtype=torch.int32)
    for bad in (lambda: hot.RelBias(table, bounds.to("meta")), lambda: hot.RelBias(meta(4, 8), bounds),
                lambda: hot.NewItems(off, 4, 4, last=i32.to("meta")), lambda: hot.NewItems(off, 4, 4, positions=i32.to("meta")),
                lambda: hot.NewItems(off.to("meta"), 4, 4, last=i32)):
        with pytest.raises(ValueError, match="on meta"):
            bad()
    b, there = hot.RelBias(table, bounds), hot.RelBias(meta(4, 8), bounds.to("meta"))
    s, x, lse, dtable = hot.SeqBatch(off, off, 4, 4, 4, 4), torch.zeros(4, 4, 8), torch.zeros(4, 4), torch.zeros(4, 8)
    elsewhere = hot.SeqBatch(off.to("meta"), off.to("meta"), 4, 4, 4, 4)
    pool = torch.zeros(2, 8, 4, 16, 8)
    c, lens, items = hot.KvCache(pool[0], pool[1], torch.zeros(1, 2, dtype=torch.int32)), torch.zeros(1, dtype=torch.int32), hot.NewItems(off, 4, 4)
    c2 = hot.KvCache(pool[0].to("meta"), pool[1].to("meta"), torch.zeros(1, 2, dtype=torch.int32, device="meta"))
    one, far = torch.zeros(1, 4, 8), hot.NewItems(off.to("meta"), 4, 4)
    for bad in (lambda: hot.dlrm_seq_attn_bias_fwd(s, there, x, x, x, x), lambda: hot.dlrm_seq_attn_bias_fwd(elsewhere, b, x, x, x, x),
                lambda: hot.dlrm_seq_attn_bias_bwd(s, there, x, x, x, x, lse, x, x, x, x, dtable, None),
                lambda: hot.dlrm_seq_attn_bias_bwd(elsewhere, b, x, x, x, x, lse, x, x, x, x, dtable, None),
                lambda: hot.dlrm_cache_attn_bias(c, lens, 32, there, one, one, None), lambda: hot.dlrm_cache_attn_bias(c, lens.to("meta"), 32, b, one, one, None),
                lambda: hot.dlrm_cache_attn_bias(c2, lens, 32, b, one, one, None), lambda: hot.dlrm_cache_tree_attn(c2, lens, 32, items, x, x, x, x, None),
                lambda: hot.dlrm_cache_tree_attn(c, lens.to("meta"), 32, items, x, x, x, x, None),
                lambda: hot.dlrm_cache_tree_attn(c, lens, 32, far, x, x, x, x, None), lambda: hot.dlrm_cache_tree_attn(c, lens, 32, items, x, x, x, x, None, bias=there)):
        with pytest.raises(ValueError, match="on meta"):
            bad()


def test_the_last_bucket_begins_where_it_is_said_to():
    """At `far`, wherever as many bounds one after the other do not pass it; of either sign, and up to the largest integer."""
    for m in range(2, 128):
        for far in [*range(m + m, 700), 2041, 4096, 10 ** 6, 2 ** 31 - 1]:
            b = hot.relative_bounds(m + 1, far).tolist()
            assert b[-1] == far and all(x < y for x, y in zip(b, b[1:])), (m, far, b)
    for n in (9, 32, 33, 128):
        for far in (200, 233, 2043, 2 ** 31 - 1):
            b = hot.relative_bounds(n, far, True).tolist()
            assert b[-1] == far and b[0] == 1 - far, (n, far, b)
    assert hot.relative_bounds(5, 2).tolist() == [1, 2, 3, 4]
