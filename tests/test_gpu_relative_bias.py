"""Attention over sequences with a learned relative position bias (dlrm_seq_attn_bias_*) against a plain 64-bit form (bias_ref), with
elementwise bounds."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from history_ref import close, offsets

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g).to(dtype)


def placed(x, layout):
    """x [T, H, d] on the device, in one of the layouts that a caller may have; what lies between the rows is NaN."""
    T, H, d = x.shape
    if layout == "rows":
        return x.to(DEV)
    if layout == "packed":      # heads side by side with others in a wider row
        v = torch.full((T, H + 3, d), NAN, dtype=x.dtype, device=DEV)[:, 1:1 + H]
    elif layout == "heads":     # head by head
        v = torch.full((H, T, d), NAN, dtype=x.dtype, device=DEV).transpose(0, 1)
    else:                       # "wide": rows wider than d
        v = torch.full((T, H, d + 8), NAN, dtype=x.dtype, device=DEV)[..., :d]
    v.copy_(x)
    return v


def bounds_of(kind, n):
    if n == 1:
        return None
    if kind == "one by one":
        return torch.arange(1, n, dtype=torch.int32)
    if kind == "both":
        return hot.relative_bounds(n, 60, True)
    if kind == "log":
        return hot.relative_bounds(n, 500)
    if kind == "far":   # every distance in the first bucket but the last ones
        return torch.arange(2 ** 31 - n, 2 ** 31 - 1, dtype=torch.int64).to(torch.int32)
    if kind == "edges":  # the ends of the integers' range, and zero
        return torch.tensor([-2 ** 31, -7, 0, 2 ** 31 - 1][:n - 1], dtype=torch.int64).to(torch.int32)
    return torch.tensor(kind, dtype=torch.int32)


LONG = [700, 40, 1100]
CASES = [
    # type, query heads, key heads, d, lengths, key lengths (None: the same), causal, prefix, slopes, cap, buckets, bounds, where the rows lie
    ("f32", 2, 2, 16, [5, 0, 1, 20, 3], None, True, False, False, 0.0, 8, "log", "rows"),
    ("f32", 4, 2, 64, [33, 64, 1, 31], None, True, False, False, 0.0, 32, "one by one", "packed"),
    ("f32", 6, 3, 72, [100, 257, 2], None, True, True, False, 0.0, 33, "both", "heads"),
    ("f32", 5, 1, 128, [70, 33], [10, 200], False, False, False, 0.0, 5, "edges", "wide"),
    ("f32", 3, 3, 96, [65, 129], None, True, False, True, 30.0, 128, "one by one", "rows"),
    ("f32", 2, 2, 40, [300] * 5, [290] * 5, True, False, False, 0.0, 16, "log", "packed"),
    ("f32", 4, 4, 64, [1300, 1200], None, True, False, False, 0.0, 64, "log", "rows"),
    ("bf16", 4, 4, 64, [200, 1, 0, 77, 130], None, True, False, False, 0.0, 32, "log", "packed"),
    ("bf16", 4, 4, 64, [200, 1, 0, 77, 130], None, False, False, False, 0.0, 32, "both", "heads"),
    ("bf16", 8, 2, 128, [90, 300], None, True, False, False, 20.0, 20, "log", "rows"),
    ("bf16", 16, 4, 128, LONG, None, True, False, False, 30.0, 64, "log", "packed"),
    ("bf16", 2, 1, 96, LONG, None, True, True, True, 0.0, 17, "both", "wide"),
    ("bf16", 3, 3, 8, [64, 63, 65, 32, 96], None, True, False, False, 0.0, 2, [1], "rows"),
    ("bf16", 33, 1, 32, [40, 7], None, True, False, False, 0.0, 7, "one by one", "packed"),
    ("bf16", 2, 2, 64, [50, 9], None, True, False, False, 0.0, 1, None, "rows"),
    ("bf16", 4, 2, 64, [150, 20], None, True, False, False, 200.0, 12, "log", "rows"),
    ("f16", 8, 2, 40, [1, 40, 17], [1000, 0, 333], False, False, False, 0.0, 32, "both", "packed"),
    ("f16", 4, 4, 64, [250, 30], None, True, False, False, 0.0, 4, "far", "rows"),
    ("f16", 2, 2, 128, LONG, None, True, False, False, 0.0, 100, "log", "heads"),
    ("f16", 1, 1, 128, [2, 1], [2600, 1500], True, False, False, 0.0, 50, "log", "rows"),
    ("f16", 8, 4, 96, [300, 301], [120, 500], True, True, False, 10.0, 31, "both", "wide"),
    ("bf16", 2, 2, 32, [0] * 40 + [600, 3] + [0] * 40, None, True, False, False, 0.0, 9, "log", "rows"),   # few of many sequences have rows
    ("bf16", 1, 1, 64, [520, 300], [100, 90], True, False, False, 0.0, 8, "log", "packed"),              # queries before the first key see none
    # enough rows for two tiles of keys a step, and for the cuts of fp32 between few rows and many
    ("bf16", 8, 4, 64, [300, 270] * 16, None, True, False, True, 0.0, 40, "log", "packed"),
    ("f16", 8, 8, 40, [290] * 30, [280, 310, 257] * 10, False, False, False, 20.0, 60, "both", "rows"),
    ("bf16", 16, 4, 128, [300, 130, 290] * 5, None, True, True, False, 0.0, 128, "one by one", "rows"),
    ("bf16", 16, 2, 104, [280, 300] * 4, None, True, False, False, 30.0, 64, "log", "rows"),
    ("f32", 8, 2, 32, [300] * 30, None, True, False, False, 0.0, 33, "both", "packed"),
    ("f32", 2, 1, 24, [3, 2, 1], [700, 900, 640], False, False, False, 5.0, 90, "both", "rows"),
]


def setup(i):
    dt, Hq, Hk, d, lens, klens, causal, prefix, slopes, cap, n, kind, where = CASES[i]
    print("[case]", i, CASES[i], flush=True)
    g, dt = gen(900 + i), DT[dt]
    klens = lens if klens is None else klens
    qo, ko, T, Tk = offsets(lens), offsets(klens), sum(lens), sum(klens)
    x = {"q": rand(g, T, Hq, d, dtype=dt), "k": rand(g, Tk, Hk, d, dtype=dt), "v": rand(g, Tk, Hk, d, dtype=dt), "do": rand(g, T, Hq, d, dtype=dt)}
    table, bounds = rand(g, Hq, n), bounds_of(kind, n)
    sl = torch.rand(Hq, generator=g) * 0.2 if slopes else None
    pre = torch.tensor([m // 4 for m in klens], dtype=torch.int32) if prefix else None
    up = lambda t: None if t is None else t.to(DEV)
    seq = hot.SeqBatch(qo.to(DEV), ko.to(DEV), T, Tk, max(lens), max(klens), causal=causal, prefix=up(pre), slopes=up(sl), cap=cap)
    return x, (qo, ko, causal, pre, sl, table, bounds, d ** -0.5, cap), seq, hot.RelBias(table.to(DEV), up(bounds)), where


def run(x, seq, bias, where, lse=True):
    dev = {n: placed(t, where) for n, t in x.items()}
    Hq, Hk, d = x["q"].shape[1], x["k"].shape[1], x["q"].shape[2]
    r = {"out": placed(torch.full_like(x["q"], NAN), where), "lse": torch.full((Hq, seq.Tq), NAN, device=DEV),
         "dq": placed(torch.full_like(x["q"], NAN), where), "dk": placed(torch.full_like(x["k"], NAN), where),
         "dv": placed(torch.full_like(x["k"], NAN), where), "dtable": torch.full_like(bias.table, NAN)}
    hot.dlrm_seq_attn_bias_fwd(seq, bias, dev["q"], dev["k"], dev["v"], r["out"], r["lse"])
    ws = hot.alloc_seq_attn_bias_workspace(seq, bias, Hq, Hk, d, binding_dtype(x["q"].dtype))
    ws.fill_(255)   # (NaN, whatever is read of it before it is written)
    hot.dlrm_seq_attn_bias_bwd(seq, bias, dev["q"], dev["k"], dev["v"], r["out"], r["lse"], dev["do"], r["dq"], r["dk"], r["dv"], r["dtable"], ws)
    return r


def binding_dtype(t):
    return {torch.float32: hot.F32, torch.float16: hot.F16, torch.bfloat16: hot.BF16}[t]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_and_gradients(i):
    x, how, seq, bias, where = setup(i)
    got = run(x, seq, bias, where)
    want = ref.attention(x["q"], x["k"], x["v"], *how, dout=x["do"])
    for n in got:
        close(got[n], want[n], want[n + "_tol"], n)
    again = run(x, seq, bias, where)
    assert all(torch.equal(got[n].nan_to_num(), again[n].nan_to_num()) for n in got)   # the same bits every time


def test_a_bias_of_zero_is_no_bias():
    """Against dlrm_seq_attn_*, whose wavefronts hold other rows: equal up to the order of fp32 sums."""
    x, (qo, ko, *_), _, bias, _ = setup(1)
    seq = hot.SeqBatch(qo.to(DEV), ko.to(DEV), int(qo[-1]), int(ko[-1]), 64, 64)
    bias.table.zero_()
    got = run(x, seq, bias, "rows")
    dev = {n: t.to(DEV) for n, t in x.items()}
    out, lse = torch.empty_like(dev["q"]), torch.empty_like(got["lse"])
    dq, dk, dv = (torch.empty_like(dev[n]) for n in "qkv")
    hot.dlrm_seq_attn_fwd(seq, dev["q"], dev["k"], dev["v"], out, lse)
    hot.dlrm_seq_attn_bwd(seq, dev["q"], dev["k"], dev["v"], out, lse, dev["do"], dq, dk, dv, hot.alloc_seq_attn_workspace(seq, 4, 2, 64))
    for a, b in ((got["out"], out), (got["lse"], lse), (got["dq"], dq), (got["dk"], dk), (got["dv"], dv)):
        assert float((a - b).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_bias_of_minus_infinity_hides_its_bucket(dtype):
    """Distances 0 and 3 to 9 hidden: the first item of a history sees nothing, and has zeros and no gradients."""
    g, dt, lens = gen(5), DT[dtype], [1, 30, 80]
    x = {n: rand(g, 111, 2, 32, dtype=dt) for n in ("q", "k", "v", "do")}
    table, bounds = rand(g, 2, 4), torch.tensor([1, 3, 10], dtype=torch.int32)
    table[:, 0] = table[0, 2] = -math.inf
    off = offsets(lens)
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), 111, 111, 80, 80)
    got = run(x, seq, hot.RelBias(table.to(DEV), bounds.to(DEV)), "rows")
    want = ref.attention(x["q"], x["k"], x["v"], off, off, True, None, None, table, bounds, 32 ** -0.5, 0.0, x["do"])
    for n in got:
        close(got[n], want[n], want[n + "_tol"], n)
    for at in (0, 1, 31):
        assert not got["out"][at].any() and not got["dq"][at].any() and torch.equal(got["lse"][:, at].cpu(), torch.full((2,), -math.inf))
    assert not got["dtable"][:, 0].any() and not got["dtable"][0, 2].any()


def test_values_of_other_sequences_do_not_matter():
    """Infinities and NaN in the rows before a sequence's, and in the sequence after it, reach none of its results."""
    g = gen(8)
    x = {n: rand(g, 68, 2, 16) for n in ("q", "k", "v", "do")}
    table, bounds = rand(g, 2, 6), torch.tensor([1, 2, 5, 9, 14], dtype=torch.int32)
    bias = hot.RelBias(table.to(DEV), bounds.to(DEV))
    plan = lambda *at: hot.SeqBatch(torch.tensor(at, device=DEV), torch.tensor(at, device=DEV), at[-1], at[-1], 45, 45)
    one = run({n: t[3:23].contiguous() for n, t in x.items()}, plan(0, 20), bias, "rows")
    for t in x.values():
        t[:3], t[23:30], t[30:] = NAN, NAN, math.inf
    two = run({n: t for n, t in x.items()}, plan(0, 3, 23, 68), bias, "rows")
    for n in ("out", "dq", "dk", "dv"):
        assert torch.equal(two[n][3:23], one[n]), n
    assert torch.equal(two["lse"][:, 3:23], one["lse"])


def test_empty_batches_write_the_table_s_gradient():
    b = hot.RelBias(torch.randn(2, 5, device=DEV), torch.arange(1, 5, dtype=torch.int32, device=DEV))
    for lens, klens in (([0, 0], [0, 0]), ([4, 0], [0, 0]), ([0, 0], [7, 3]), ([0, 5], [6, 0])):
        qo, ko = offsets(lens).to(DEV), offsets(klens).to(DEV)
        T, Tk = sum(lens), sum(klens)
        seq = hot.SeqBatch(qo, ko, T, Tk, max(max(lens), 1), max(max(klens), 1), causal=False)
        x = {n: torch.randn(T if n in ("q", "do") else Tk, 2, 8) for n in ("q", "k", "v", "do")}
        got = run(x, seq, b, "rows")
        assert torch.equal(got["dtable"], torch.zeros_like(b.table)), (lens, klens)
        assert not got["out"].any() and not got["dq"].any() and not got["dk"].any() and not got["dv"].any()


def test_the_tables_gradient_against_differences():
    """Of the kernels' own forward, fp32: a step of 2^-6 either way; the forward's rounding and the third derivative stay below 1e-3 of the largest."""
    g, lens = gen(31), [50, 90, 3]
    off, T = offsets(lens), 143
    x = {n: rand(g, T, 2, 16) for n in ("q", "k", "v", "do")}
    bounds = torch.tensor([1, 4, 30], dtype=torch.int32, device=DEV)
    table = rand(g, 2, 4).to(DEV)
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 90, 90)
    dtable = run(x, seq, hot.RelBias(table, bounds), "rows")["dtable"].double()
    dev = {n: t.to(DEV) for n, t in x.items()}

    def loss(t):
        out = torch.empty_like(dev["q"])
        hot.dlrm_seq_attn_bias_fwd(seq, hot.RelBias(t, bounds), dev["q"], dev["k"], dev["v"], out)
        return float((out.double() * dev["do"].double()).sum())
    step = 2.0 ** -6
    for h in range(2):
        for b in range(4):
            t = [table.clone(), table.clone()]
            t[0][h, b] += step
            t[1][h, b] -= step
            assert abs((loss(t[0]) - loss(t[1])) / (2 * step) - float(dtable[h, b])) < 1e-3 * float(dtable.abs().max())


def test_many_sequences_of_uneven_lengths():
    """Blocks laid one sequence after the other (few of them are long), every wavefront's sums of the table's gradient joined in two steps."""
    g = gen(41)
    lens = [0, 3, 1] * 400 + [900] + [2] * 500 + [70]
    off, T = offsets(lens), sum(lens)
    x = {n: rand(g, T, 2, 16, dtype=torch.bfloat16) for n in ("q", "k", "v", "do")}
    table, bounds = rand(g, 2, 24), hot.relative_bounds(24, 200)
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 900, 900)
    got = run(x, seq, hot.RelBias(table.to(DEV), bounds.to(DEV)), "rows")
    want = ref.attention(x["q"], x["k"], x["v"], off, off, True, None, None, table, bounds, 0.25, 0.0, x["do"])
    for n in got:
        close(got[n], want[n], want[n + "_tol"], n)


def test_a_graph_of_forward_and_backward_replays_like_eager_calls():
    g, lens = gen(51), [40, 3, 130]
    off, T = offsets(lens).to(DEV), sum(lens)
    seq = hot.SeqBatch(off, off, T, T, 130, 130)
    bias = hot.RelBias(torch.randn(4, 32, device=DEV), hot.relative_bounds(32, 100, device=DEV))
    mk = lambda H: torch.empty(T, H, 64, dtype=torch.bfloat16, device=DEV)
    q, k, v, do, out, dq, dk, dv = (mk(H) for H in (4, 2, 2, 4, 4, 4, 2, 2))
    lse, dtable, ws = torch.empty(4, T, device=DEV), torch.empty(4, 32, device=DEV), hot.alloc_seq_attn_bias_workspace(seq, bias, 4, 2, 64)

    def step():
        hot.dlrm_seq_attn_bias_fwd(seq, bias, q, k, v, out, lse)
        hot.dlrm_seq_attn_bias_bwd(seq, bias, q, k, v, out, lse, do, dq, dk, dv, dtable, ws)

    def fill():
        for x in (q, k, v, do):
            x.copy_(rand(g, *x.shape, dtype=torch.bfloat16))
        bias.table.copy_(rand(g, 4, 32))
    fill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        fill()
        graph.replay()
        got = [x.clone() for x in (out, lse, dq, dk, dv, dtable)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, dq, dk, dv, dtable)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("lowest", [torch.finfo(torch.float32).min, -1e9, torch.finfo(torch.float16).min, -60000.0])
def test_the_lowest_numbers_hide_their_buckets_too(lowest):
    """As -inf does: a row of nothing else has zeros, and no gradients; the greatest number that does not hide is a bias."""
    g, lens = gen(6), [1, 30, 80]
    x = {n: rand(g, 111, 2, 32) for n in ("q", "k", "v", "do")}
    bounds, off = torch.tensor([1, 3, 10], dtype=torch.int32), offsets(lens)
    table = rand(g, 2, 4)
    table[:, 0] = table[0, 2] = lowest
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), 111, 111, 80, 80)
    got = run(x, seq, hot.RelBias(table.to(DEV), bounds.to(DEV)), "rows")
    hidden = torch.where(table <= -60000.0, torch.full_like(table, -math.inf), table)
    want = ref.attention(x["q"], x["k"], x["v"], off, off, True, None, None, hidden, bounds, 32 ** -0.5, 0.0, x["do"])
    for n in got:
        close(got[n], want[n], want[n + "_tol"], n)
    assert not got["dtable"][:, 0].any() and not got["out"][0].any()


def test_bounds_that_do_not_ascend_stay_within_the_table():
    """What they mean is not said; every pair has some bucket of the table, and results are finite."""
    g = gen(7)
    off = offsets([90, 200])
    x = {n: rand(g, 290, 2, 16, dtype=torch.bfloat16) for n in ("q", "k", "v", "do")}
    bounds = torch.tensor([9, 3, 3, 150, -40, 20, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).to(torch.int32)
    bias = hot.RelBias(rand(g, 2, 9).to(DEV), bounds.to(DEV))
    got = run(x, hot.SeqBatch(off.to(DEV), off.to(DEV), 290, 290, 200, 200, causal=False), bias, "rows")
    assert all(torch.isfinite(t).all() for t in got.values())


def test_calls_on_two_streams_at_once_are_what_they_are_alone():
    """Each with a workspace of its own, on streams other than the tensors'."""
    g, lens = gen(52), [400, 3, 130, 257]
    off, T = offsets(lens).to(DEV), sum(lens)
    seq = hot.SeqBatch(off, off, T, T, 400, 400)
    bias = hot.RelBias(torch.randn(4, 32, device=DEV), hot.relative_bounds(32, 100, device=DEV))
    heads = (4, 2, 2, 4)
    x = [[rand(g, T, H, 64, dtype=torch.bfloat16).to(DEV) for H in heads] for _ in range(2)]

    def step(i, out, lse, dq, dk, dv, dtable, ws):
        q, k, v, do = x[i]
        hot.dlrm_seq_attn_bias_fwd(seq, bias, q, k, v, out, lse)
        hot.dlrm_seq_attn_bias_bwd(seq, bias, q, k, v, out, lse, do, dq, dk, dv, dtable, ws)

    def room():
        mk = lambda H: torch.empty(T, H, 64, dtype=torch.bfloat16, device=DEV)
        return mk(4), torch.empty(4, T, device=DEV), mk(4), mk(2), mk(2), torch.empty(4, 32, device=DEV), hot.alloc_seq_attn_bias_workspace(seq, bias, 4, 2, 64)
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
        for y, z in zip(a[:-1], b[:-1]):
            assert torch.equal(y, z)
