"""Operators that read a history in order where their arguments end: strides, lengths, grids and values at the edge of what a call takes.
Values against the plain 64-bit forms of history_ref with its bounds; a tighter bound is derived where it stands."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def hand_memory_back():
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def far_apart(n, H, d, stride, dtype, tensors=1):
    """Views [n, H, d] whose items lie `stride` elements apart, the views' rows side by side; what lies between is not touched."""
    assert tensors * H * d <= stride
    pool = torch.empty((n - 1) * stride + tensors * H * d, dtype=dtype, device=DEV)
    return [pool[i * H * d:].as_strided((n, H, d), (stride, d, 1), i * H * d) for i in range(tensors)]


# ------------------------------------------------------------------------------------------------ strides
@pytest.mark.parametrize("dtype,d,stride,slopes", [("f32", 16, 1 << 23, False), ("f32", 64, (1 << 22) + 8, True), ("f16", 64, 1 << 23, False), ("f32", 72, 1 << 22, False)])
def test_keys_a_large_stride_apart(dtype, d, stride, slopes):
    """Few queries over some hundred keys whose rows lie up to the largest stride apart: every row that a tile takes is its own."""
    g, dt, nq, nk, H = gen(d), DT[dtype], 3, 520, 2
    q, do = (rand(g, nq, H, d, dtype=dt) for _ in range(2))
    k, v = (rand(g, nk, H, d, dtype=dt) for _ in range(2))
    K, V, DK, DV = far_apart(nk, H, d, stride, dt, 4)
    K.copy_(k)
    V.copy_(v)
    Q, DO, DQ, O = far_apart(nq, H, d, stride, dt, 4)
    Q.copy_(q)
    DO.copy_(do)
    qo, ko = torch.tensor([0, nq], device=DEV), torch.tensor([0, nk], device=DEV)
    sl = torch.tensor([0.01, 0.0]) if slopes else None
    seq = hot.SeqBatch(qo, ko, nq, nk, nq, nk, slopes=None if sl is None else sl.to(DEV))
    lse = torch.empty(H, nq, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, O, lse)
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, O, lse, DO, DQ, DK, DV, hot.alloc_seq_attn_workspace(seq, H, H, d))
    want = ref.attention(q, k, v, qo.cpu(), ko.cpu(), True, None, sl, d ** -0.5, 0.0, do)
    for n, x in (("out", O), ("lse", lse), ("dq", DQ), ("dk", DK), ("dv", DV)):
        ref.close(x, want[n], want[n + "_tol"], n)


# ------------------------------------------------------------------------------------------------ columns that are not rotated
def bits(x):
    return x.contiguous().view(torch.int32 if x.dtype == torch.float32 else torch.int16)


@pytest.mark.parametrize("layout", [hot.ROPE_HALF, hot.ROPE_INTERLEAVED])
@pytest.mark.parametrize("dtype,d,rot", [("f32", 16, 0), ("f16", 72, 20), ("bf16", 72, 64), ("bf16", 128, 0), ("f32", 40, 6), ("f16", 64, 32), ("bf16", 16, 16)])
def test_columns_past_the_rotated_ones_keep_every_value(dtype, d, rot, layout):
    """Without a norm they are copied, forward and backward, whatever they hold and whatever their neighbours hold."""
    dt, T, Hq, Hk = DT[dtype], 40, 3, 2
    g = gen(d + rot)
    x = [rand(g, T, H, d, dtype=dt) for H in (Hq, Hk)]
    odd = torch.tensor([INF, -INF, NAN, -0.0, 0.0, torch.finfo(dt).max, torch.finfo(dt).tiny], dtype=dt)
    for t in x:
        at = torch.rand(t.shape, generator=g) < 0.3
        at[..., :rot] = False                      # (rotated columns are finite: what they become has to stay so)
        t[at] = odd[torch.randint(0, len(odd), (int(at.sum()),), generator=g)]
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    plan = hot.QkRope(pos, Hq, Hk, d, inv_freq=hot.rope_frequencies(rot, device=DEV) if rot else None, rot=rot, layout=layout, mscale=1.5)
    X = [t.to(DEV) for t in x]
    fwd, bwd = ([torch.zeros_like(t) for t in X] for _ in range(2))
    hot.dlrm_qk_rope_fwd(plan, X[0], X[1], fwd[0], fwd[1])
    hot.dlrm_qk_rope_bwd(plan, X[0], X[1], X[0], X[1], bwd[0], bwd[1], None, None, None)
    for a, b, c in zip(x, fwd, bwd):
        nan = a[..., rot:].isnan()                 # (of a NaN only that it is one)
        for y in (b.cpu(), c.cpu()):
            assert torch.equal(y[..., rot:].isnan(), nan)
            assert torch.equal(bits(y[..., rot:])[~nan], bits(a[..., rot:])[~nan])
            assert torch.isfinite(y[..., :rot]).all()


@pytest.mark.parametrize("layout", [hot.ROPE_HALF, hot.ROPE_INTERLEAVED])
def test_an_infinite_column_of_a_gradient_stays_in_its_column(layout):
    """With a norm: dy infinite in a column past the rotated ones makes its row's mean infinite, so the row; no other row, and dw in its column alone."""
    g, T, d, rot = gen(3), 9, 32, 8
    x, dy = rand(g, T, 1, d), rand(g, T, 1, d)
    dy[4, 0, 21] = INF
    w = 1 + 0.1 * rand(g, d)
    plan = hot.QkRope(torch.arange(T, dtype=torch.int32, device=DEV), 1, 0, d, inv_freq=hot.rope_frequencies(rot, device=DEV), wq=w.to(DEV), layout=layout)
    dx, dw = torch.zeros(T, 1, d, device=DEV), torch.zeros(d, device=DEV)
    hot.dlrm_qk_rope_bwd(plan, x.to(DEV), None, dy.to(DEV), None, dx, None, dw, None, hot.alloc_qk_rope_workspace(plan))
    rows, cols = torch.arange(T) != 4, torch.arange(d) != 21
    assert torch.isfinite(dx.cpu()[rows]).all() and torch.isfinite(dw.cpu()[cols]).all()
    assert float(dw[21]) == math.copysign(INF, float(x[4, 0, 21]))


# ------------------------------------------------------------------------------------------------ the longest caches
@pytest.mark.parametrize("page,cols,last", [(1024, (1 << 21) - 1, 1100), (1, (1 << 31) - 1, 700), (128, 1 << 23, 5)])
def test_the_last_chunk_of_a_cache_of_two_billion_items(page, cols, last):
    """One sequence whose table names the same two pages again and again: page 1 for the `last` columns, page 0 for all before.  The last ones' keys
    carry half of the weight, so a chunk that is left out shows.  (128 x 2^23 items: 2^30, a length that divides.)"""
    g, dt, H, d = gen(cols % 97), torch.float16, 1, 8
    k, v = (rand(g, 2, H, page, d, dtype=dt) for _ in range(2))
    k[..., 0] = 0.0
    q = torch.zeros(1, H, d, dtype=dt)
    q[0, 0, 0] = 1.0                                           # the score is scale times the key's first column
    n = [(cols - last) * page, last * page]
    k[1, :, :, 0] = math.log(n[0] / n[1])                      # (rounded to the type: the reference takes what it became)
    v[1] += 4.0
    table = torch.zeros(1, cols, dtype=torch.int32, device=DEV)
    table[0, -last:] = 1
    cache = hot.KvCache(k.to(DEV), v.to(DEV), table)
    held = cols * page
    out = torch.full((1, H, d), NAN, dtype=dt, device=DEV)
    hot.dlrm_cache_attn(cache, torch.tensor([held], dtype=torch.int32, device=DEV), held, q.to(DEV), out, hot.alloc_cache_attn_workspace(cache, H, held), scale=1.0)
    sc = k[:, 0, :, 0].double()                                # [page 0 or 1, item]
    w = torch.exp(sc - sc.max()) * torch.tensor(n, dtype=torch.float64)[:, None] / page
    p = w / w.sum()
    want, mags = (p[..., None] * v[:, 0].double()).sum((0, 1)), (p[..., None] * v[:, 0].double().abs()).sum((0, 1))
    # fp32 sums: a lane adds 8 weights a step, a chunk of 2^20 keys is 8192 steps of its four wavefronts, and a sequence up to 2^21 chunks
    # that 512 threads add: at most 2^16 + 2^12 + 600 roundings on any path, in numerator and denominator each; the type's two roundings
    tol = ref.UNIT[dt] * want.abs() + (ref.UNIT[dt] + 2 * (2 ** 16 + 2 ** 12 + 600) * ref.E32) * mags
    ref.close(out[0, 0], want, tol, "out")
    assert float(want.min()) > 1.0                             # (half of 4: without the last chunk the values' mean is near 0)


def test_one_workspace_for_every_smaller_bound():
    """A server's workspace, allocated for its longest history, with the bound of each call."""
    g, B, Hq, Hk, d, page, top = gen(19), 8, 16, 4, 128, 64, 8256
    cols = top // page
    k, v = (torch.randn(B * cols, Hk, page, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    cache = hot.KvCache(k, v, torch.randperm(B * cols, generator=g).to(torch.int32).view(B, cols).to(DEV))
    q = rand(g, B, Hq, d, dtype=torch.bfloat16).to(DEV)
    ws = hot.alloc_cache_attn_workspace(cache, Hq, top)
    for n in (8000, 8256, 1, 300, 4100, 8192):
        lens, out, own = torch.full((B,), n, dtype=torch.int32, device=DEV), torch.empty_like(q), torch.empty_like(q)
        hot.dlrm_cache_attn(cache, lens, n, q, out, ws)
        hot.dlrm_cache_attn(cache, lens, n, q, own, hot.alloc_cache_attn_workspace(cache, Hq, n))
        assert torch.equal(out, own) and torch.isfinite(out).all()


# ------------------------------------------------------------------------------------------------ more threads than a launch takes
def test_more_rows_than_one_launch_has_threads_for():
    """2^28 rows of 72 bf16 columns are 2^32 lanes.  Rows and positions repeat, so the result does: it is compared, bit for bit, with a small call's."""
    d, P, T, dt = 72, 1 << 16, (1 << 28) + 70003, torch.bfloat16
    block = torch.randn(P, 1, d, device=DEV).to(dt)
    pos = (torch.arange(T, device=DEV, dtype=torch.int32) & (P - 1))
    w, f = torch.linspace(0.5, 1.5, d, device=DEV), hot.rope_frequencies(64, device=DEV)
    want = torch.empty_like(block)
    hot.dlrm_qk_rope_fwd(hot.QkRope(pos[:P], 1, 0, d, inv_freq=f, wq=w), block, None, want, None)
    x = torch.empty(T, 1, d, dtype=dt, device=DEV)
    for t in range(0, T, P):
        x[t:t + P] = block[:min(P, T - t)]
    hot.dlrm_qk_rope_fwd(hot.QkRope(pos, 1, 0, d, inv_freq=f, wq=w), x, None, x, None)
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for t in range(0, T, P):
        bad += (x[t:t + P] != want[:min(P, T - t)]).any()
    assert int(bad) == 0


def test_more_appended_items_than_one_launch_has_threads_for():
    """2^28 items of one query, key and value of 72 bf16 columns, in sequences of 64.  The first and the last thousand sequences have pages, the others none."""
    d, n_items, dt, page = 72, (1 << 28) + 6400, torch.bfloat16, 64
    B = n_items // page
    x = torch.randn(n_items, 1, 1, dtype=dt, device=DEV).expand(n_items, 1, 8).repeat(1, 1, 9)       # every row one value
    pos = torch.arange(n_items, device=DEV, dtype=torch.int32) & (page - 1)
    seqs = (torch.arange(n_items, device=DEV, dtype=torch.int32) >> 6)
    table = torch.full((B, 1), -1, dtype=torch.int32, device=DEV)
    table[:1000, 0] = torch.arange(1000, device=DEV, dtype=torch.int32)
    table[-1000:, 0] = torch.arange(1000, 2000, device=DEV, dtype=torch.int32)
    pool = torch.full((2, 2000, 1, page, d), 7.0, dtype=dt, device=DEV)
    plan = hot.QkRope(pos, 1, 1, d)
    q = torch.zeros(n_items, 1, d, dtype=dt, device=DEV)
    hot.dlrm_qk_rope_append(plan, q, x, x, q, hot.KvCache(pool[0], pool[1], table), seqs)
    for half, rows in ((slice(0, 1000), x[:64000]), (slice(1000, 2000), x[-64000:])):
        for p in pool:
            assert torch.equal(p[half].reshape(-1, 1, d), rows)


@pytest.mark.parametrize("B,top,page,Hq,Hk,slopes", [((1 << 21) + 301, 512, 512, 8, 8, False), ((1 << 23) + 301, 16, 16, 8, 8, True), ((700 << 10) + 77, 2100, 1, 24, 8, False)])
def test_more_sequences_than_one_launch_has_threads_for(B, top, page, Hq, Hk, slopes):
    """Of four wavefronts each, of one, and in three chunks with a join.  Queries, lengths and tables repeat, so the result does: it is compared with a
    small call's."""
    g, d, P, dt, cols = gen(B % 1000), 8, 4096, torch.bfloat16, (top + page - 1) // page
    k, v = (torch.randn(4 * cols, Hk, page, d, device=DEV).to(dt) for _ in range(2))
    table = (torch.arange(P)[:, None] % 4 * cols + torch.arange(cols)).to(torch.int32).to(DEV)
    lens = torch.randint(0, 4, (P,), generator=g).to(torch.int32)
    lens[5::977] = top                                         # a few long ones: their walks and joins are whole
    lens = lens.to(DEV)
    q = torch.randn(P, Hq, d, device=DEV).to(dt)
    sl = torch.linspace(0.1, 1.0, Hq, device=DEV) if slopes else None
    n = (B + P - 1) // P
    cache = hot.KvCache(k, v, table.repeat(n, 1)[:B].contiguous())
    Q = q.repeat(n, 1, 1)[:B].contiguous()
    out = torch.full_like(Q, NAN)
    hot.dlrm_cache_attn(cache, lens.repeat(n)[:B].contiguous(), top, Q, out, hot.alloc_cache_attn_workspace(cache, Hq, top), slopes=sl)
    part = out[:P].float()
    for s in range(0, B, P):
        assert torch.equal(out[s:s + P], out[:min(P, B - s)])
    small = torch.empty_like(q)
    c = hot.KvCache(k, v, table)
    hot.dlrm_cache_attn(c, lens, top, q, small, hot.alloc_cache_attn_workspace(c, Hq, top), slopes=sl)
    # (the small call may be cut otherwise: fp32 sums in another order, weights rounded from another maximum, one rounding of the result)
    off = (part - small.float()).abs()
    assert float((off - 4 * ref.UNIT[dt] * v.float().abs().max()).max()) <= 0 and float(part.abs().sum()) > 0


# ------------------------------------------------------------------------------------------------ sequences: bounds
@pytest.mark.parametrize("dtype,d,Hq,Hk", [("bf16", 64, 4, 2), ("f32", 32, 2, 2)])
def test_bounds_that_say_nothing(dtype, d, Hq, Hk):
    """2^31 - 1 for both: the results of exact bounds."""
    g, dt, lens = gen(5), DT[dtype], [70, 0, 300, 1]
    off, T = ref.offsets(lens).to(DEV), sum(lens)
    q, do = (rand(g, T, Hq, d, dtype=dt).to(DEV) for _ in range(2))
    k, v = (rand(g, T, Hk, d, dtype=dt).to(DEV) for _ in range(2))
    want = ref.attention(q.cpu(), k.cpu(), v.cpu(), off.cpu(), off.cpu(), True, None, None, d ** -0.5, 0.0, do.cpu())
    for top in ((1 << 31) - 1, 300):
        seq = hot.SeqBatch(off, off, T, T, top, top)
        out, dq, dk, dv = (torch.full_like(x, NAN) for x in (q, q, k, v))
        lse = torch.empty(Hq, T, device=DEV)
        hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
        hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
        for n, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            ref.close(x, want[n], want[n + "_tol"], n)


@pytest.mark.parametrize("dtype,B,H", [("bf16", (1 << 20) + 301, 64), ("f32", (1 << 22) + 301, 8), ("f16", (1 << 26) + 301, 1)])
def test_more_blocks_than_one_launch_has_threads_for(dtype, B, H):
    """Histories of up to two items: 2^26 workgroups of one wavefront for the keys, and as many of two or more for the queries.  Rows and lengths repeat, so
    the results do: they are compared, bit for bit, with the 64-bit form's of one round, and with each other."""
    g, dt, d, P = gen(H), DT[dtype], 8, 64
    lens = torch.randint(0, 3, (P,), generator=g)
    lens[:2] = torch.tensor([2, 1])
    n, rows = B // P, int(lens.sum())
    all_lens = torch.cat([lens.repeat(n), lens[:B - n * P]])
    off = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(all_lens, 0)]).to(DEV)
    T = int(off[-1])
    small = [rand(g, rows, H, d, dtype=dt) for _ in range(4)]
    q, k, v, do = (torch.cat([x.to(DEV).repeat(n, 1, 1), x[:T - n * rows].to(DEV)]) for x in small)
    seq = hot.SeqBatch(off, off, T, T, 2, 2)
    out, dq, dk, dv = (torch.full_like(x, NAN) for x in (q, q, k, v))
    lse = torch.full((H, T), NAN, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
    hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, H, H, d))
    o = ref.offsets(lens.numpy())
    want = ref.attention(*small[:3], o, o, True, None, None, d ** -0.5, 0.0, small[3])
    for name, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv), ("lse", lse.t())):
        one = x[:rows]
        if name != "lse":
            ref.close(one, want[name], want[name + "_tol"], name)
        else:
            ref.close(one.t(), want[name], want[name + "_tol"], name)
        whole = x[:n * rows].reshape(n, rows, *x.shape[1:])
        for a in range(0, n, 1 << 14):
            assert (whole[a:a + (1 << 14)] == one).all(), (name, a)
        assert torch.equal(x[n * rows:], one[:T - n * rows]), name


@pytest.mark.parametrize("dtype,causal", [("f32", True), ("f32", False), ("bf16", True)])
def test_distances_past_the_integers_of_fp32(dtype, causal):
    """70 queries at the end of 2^24 + 6001 keys, slopes of 1/2 and 1/4: only the last keys weigh anything, and their distances are those of a short sequence."""
    g, dt, nq, nk, H, d, last = gen(24), DT[dtype], 70, (1 << 24) + 6001, 2, 8, 4096
    q, do = (rand(g, nq, H, d, dtype=dt) for _ in range(2))
    k, v = (torch.randn(nk, H, d, device=DEV).to(dt) for _ in range(2))
    sl = torch.tensor([0.5, 0.25])
    seq = hot.SeqBatch(torch.tensor([0, nq], device=DEV), torch.tensor([0, nk], device=DEV), nq, nk, nq, nk, causal=causal, slopes=sl.to(DEV))
    Q, DO = q.to(DEV), do.to(DEV)
    out, dq, dk, dv = (torch.full_like(x, NAN) for x in (Q, Q, k, v))
    lse = torch.empty(H, nq, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, k, v, out, lse)
    hot.dlrm_seq_attn_bwd(seq, Q, k, v, out, lse, DO, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, H, H, d))
    want = ref.attention(q, k[-last:].cpu(), v[-last:].cpu(), torch.tensor([0, nq]), torch.tensor([0, last]), causal, None, sl, d ** -0.5, 0.0, do)
    for n, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk[-last:]), ("dv", dv[-last:])):
        ref.close(x, want[n], want[n + "_tol"], n)
    assert not dk[:-last].any() and not dv[:-last].any()


@pytest.mark.parametrize("dtype,d,n", [("f32", 32, 40), ("f16", 64, 40), ("bf16", 128, 40), ("bf16", 16, 700), ("f32", 96, 700)])
@pytest.mark.parametrize("what", [NAN, INF])
def test_a_query_that_is_not_finite_does_not_pass_for_one_that_sees_nothing(dtype, d, n, what):
    """Its weights are NaN: so are its row, its lse and the gradients of the values that it sees, and nobody else's rows."""
    g, dt, i = gen(d), DT[dtype], 21
    q, k, v, do = (rand(g, n, 1, d, dtype=dt) for _ in range(4))
    q[i, 0, 3] = what
    k[:, 0, 3] = 1.0                                            # (the score is infinite or NaN, whatever the other columns give)
    off = torch.tensor([0, n], device=DEV)
    seq = hot.SeqBatch(off, off, n, n, n, n)
    x = [t.to(DEV) for t in (q, k, v)]
    out, dq, dk, dv = (torch.empty(n, 1, d, dtype=dt, device=DEV) for _ in range(4))
    lse = torch.empty(1, n, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, *x, out, lse)
    hot.dlrm_seq_attn_bwd(seq, *x, out, lse, do.to(DEV), dq, dk, dv, hot.alloc_seq_attn_workspace(seq, 1, 1, d))
    mine = torch.arange(n, device=DEV) == i
    for y in (out, dq):
        assert y[i].isnan().all() and torch.isfinite(y[~mine]).all()
    assert lse[0, i].isnan() and torch.isfinite(lse[0, ~mine]).all()
    assert dv[:i + 1].isnan().all() and torch.isfinite(dv[i + 1:]).all()
    assert dk[:i + 1].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("stride", [0, 1, 24])
def test_the_stride_of_one_item_means_nothing(dtype, stride):
    """One query over one key, whose value has an infinity: a product with rows that are not there would make it NaN."""
    g, dt, d = gen(stride), DT[dtype], 40
    rows = [rand(g, 1, 2, d, dtype=dt) for _ in range(4)]
    rows[2][0, 1, 7] = INF
    one = lambda x: x.to(DEV).as_strided((1, 2, d), (stride, d, 1))
    q, k, v, do = (one(x) for x in rows)
    out, dq, dk, dv = (one(torch.zeros(1, 2, d, dtype=dt)) for _ in range(4))
    off = torch.tensor([0, 1], device=DEV)
    seq, lse = hot.SeqBatch(off, off, 1, 1, 1, 1), torch.empty(2, 1, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
    assert torch.equal(out, v)
    hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, 2, 2, d))
    assert torch.isfinite(dv).all() and torch.isfinite(dk[:, 0]).all() and torch.isfinite(dq[:, 0]).all()
    plan = hot.QkRope(torch.zeros(1, dtype=torch.int32, device=DEV), 2, 2, d)
    qo, ko = one(torch.zeros(1, 2, d, dtype=dt)), one(torch.zeros(1, 2, d, dtype=dt))
    hot.dlrm_qk_rope_fwd(plan, q, v, qo, ko)
    assert torch.equal(qo, q) and torch.equal(ko, v)


# ------------------------------------------------------------------------------------------------ digits
def norm_off(got, want, dt):
    """Distance from the exact result in the Euclidean norm over all rows, and that of the result rounded to the type."""
    return float((got.double() - want).norm()), float((want.to(dt).double() - want).norm())


@pytest.mark.parametrize("dtype,d,cap", [("bf16", 128, 0.0), ("f16", 64, 0.0), ("bf16", 40, 30.0)])
def test_cached_attention_is_off_by_the_rounding_of_its_result(dtype, d, cap):
    """The weights' own rounding (they are taken in two parts, to 2^-16 at least) and fp32 add less than a twentieth to it: 2^-16 / 2^-9 is an eightieth, a capped
    score's 2^-16 as much again."""
    dt, B, H, page, n = DT[dtype], 40, 4, 64, 1500
    g = torch.Generator(device=DEV).manual_seed(d)
    q = torch.randn(B, H, d, generator=g, device=DEV).to(dt)
    cols = (n + page - 1) // page
    k, v = (torch.randn(B * cols, 1, page, d, generator=g, device=DEV).to(dt) for _ in range(2))
    cache = hot.KvCache(k, v, torch.arange(B * cols, dtype=torch.int32, device=DEV).view(B, cols))
    out = torch.empty_like(q)
    hot.dlrm_cache_attn(cache, torch.full((B,), n, dtype=torch.int32, device=DEV), n, q, out, hot.alloc_cache_attn_workspace(cache, H, n), cap=cap)
    K, V = (x.double().view(B, cols * page, d)[:, :n] for x in (k, v))
    x = torch.matmul(q.double(), K.transpose(1, 2).contiguous()) * d ** -0.5
    want = torch.matmul(torch.softmax(cap * torch.tanh(x / cap) if cap else x, -1), V)
    off, rounding = norm_off(out, want, dt)
    assert off <= 1.05 * rounding, (off, rounding)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 64), ("bf16", 24)])
def test_short_histories_of_narrow_rows_are_off_by_the_rounding_of_their_results(dtype, d):
    """Weights and score gradients in two parts: out, dk and dv as above.  dq's delta comes from the stored out for rows of more than 32 keys: its rounding moves ds
    by as much as rounding ds once would, at most, so dq is off by no more than two roundings of which the first is made up of."""
    dt, Hq, Hk = DT[dtype], 4, 2
    g = torch.Generator(device=DEV).manual_seed(d)
    lens = [1 + (37 * i) % 200 for i in range(40)]
    off, T = ref.offsets(lens), sum(lens)
    q, do = (torch.randn(T, Hq, d, generator=g, device=DEV).to(dt) for _ in range(2))
    k, v = (torch.randn(T, Hk, d, generator=g, device=DEV).to(dt) for _ in range(2))
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 200, 200)
    got = {n: torch.empty_like(x) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    lse = torch.empty(Hq, T, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, q, k, v, got["out"], lse)
    hot.dlrm_seq_attn_bwd(seq, q, k, v, got["out"], lse, do, got["dq"], got["dk"], got["dv"], hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
    want = {n: torch.zeros(x.shape, dtype=torch.float64, device=DEV) for n, x in got.items()}
    for s, n in enumerate(lens):
        I = slice(int(off[s]), int(off[s]) + n)
        for h in range(Hq):
            Q, K, V, D = (x.double() for x in (q[I, h], k[I, h // 2], v[I, h // 2], do[I, h]))
            x = (Q @ K.t() * d ** -0.5).masked_fill(torch.ones(n, n, device=DEV).triu(1).bool(), -math.inf)
            p = torch.softmax(x, -1)
            o = p @ V
            ds = p * (D @ V.t() - (D * o).sum(-1, keepdim=True)) * d ** -0.5
            want["out"][I, h], want["dq"][I, h] = o, ds @ K
            want["dk"][I, h // 2] += ds.t() @ Q
            want["dv"][I, h // 2] += p.t() @ D
    for n, x in got.items():
        err, rounding = norm_off(x, want[n], dt)
        assert err <= (1.42 if n == "dq" else 1.05) * rounding, (n, err, rounding)


@pytest.mark.parametrize("dtype,d", [("f32", 32), ("f16", 64), ("bf16", 128), ("f32", 96)])
def test_the_value_of_the_largest_score_by_far(dtype, d):
    """Integer queries and keys, so that every type and fp32 hold the scores exactly; in rows whose largest score leads by 200 or more the others' weights are
    below e^-200, and the row is that key's value to two roundings."""
    g, dt, n = gen(d), DT[dtype], 300
    q, k = (torch.randint(-16, 17, (n, 1, d), generator=g).to(dt) for _ in range(2))
    v = rand(g, n, 1, d, dtype=dt)
    off = torch.tensor([0, n], device=DEV)
    out, lse = torch.empty(n, 1, d, dtype=dt, device=DEV), torch.empty(1, n, device=DEV)
    hot.dlrm_seq_attn_fwd(hot.SeqBatch(off, off, n, n, n, n, scale=1.0), q.to(DEV), k.to(DEV), v.to(DEV), out, lse)
    sc = (q[:, 0].double() @ k[:, 0].double().t()).masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf)
    top = sc.topk(2, -1)
    clear = top.values[:, 0] - top.values[:, 1] >= 200
    assert int(clear.sum()) >= 50
    want = v[top.indices[:, 0], 0].double()
    # (the exponent, up to 2^16, is rounded when the maximum is taken: the weight is 2^(2^-9) off 1 at most, and stands in the sum as it is; what a
    # 16-bit weight is rounded by is u, and the result once more)
    bound = (2 * ref.UNIT[dt] + 2.0 ** -22) * want.abs() + ref.TINY[dt]
    assert ((out[:, 0].double().cpu() - want).abs() <= bound)[clear].all()
    ref.close(lse[0].cpu()[clear], top.values[:, 0][clear], 4 * ref.E32 * top.values[:, 0][clear].abs() + 1e-30, "lse")


# ------------------------------------------------------------------------------------------------ angles
def angle(position, frequency):
    """position * frequency modulo 2 pi, to 30 digits."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    two_pi = Decimal("6.28318530717958647692528676655900576839433879875021164194989")
    x = Decimal(position) * Decimal(frequency)      # (both exact)
    return float(x - (x / two_pi).to_integral_value() * two_pi)


@pytest.mark.parametrize("layout", [hot.ROPE_HALF, hot.ROPE_INTERLEAVED])
@pytest.mark.parametrize("top", [1 << 12, 1 << 24, 1 << 31])
def test_angles_of_large_positions(layout, top):
    """An angle is off by 3 2^-53 of itself (1 / 2 pi and two products in fp64) and what sine and cosine in fp32 add, 2^-22."""
    T, rot = 50, 16
    pos = [top - 1 - (7919 * i) % (top // 2) for i in range(T)]
    f = hot.rope_frequencies(rot)
    x = rand(gen(top % 1000), T, 1, rot)
    y = torch.empty(T, 1, rot, device=DEV)
    hot.dlrm_qk_rope_fwd(hot.QkRope(torch.tensor(pos, dtype=torch.int32, device=DEV), 1, 0, rot, inv_freq=f.to(DEV), layout=layout), x.to(DEV), None, y, None)
    a = torch.tensor([[angle(p, float(w)) for w in f] for p in pos], dtype=torch.float64)
    n = rot // 2
    i, j = (torch.arange(n), torch.arange(n) + n) if layout == hot.ROPE_HALF else (2 * torch.arange(n), 2 * torch.arange(n) + 1)
    u, v = x[:, 0, i].double(), x[:, 0, j].double()
    got = y[:, 0].double().cpu()
    off = 3 * 2.0 ** -53 * torch.tensor(pos, dtype=torch.float64)[:, None] * f.double() + 2.0 ** -22
    for want, at in ((u * a.cos() - v * a.sin(), i), (v * a.cos() + u * a.sin(), j)):
        assert ((got[:, at] - want).abs() <= off * (u.abs() + v.abs())).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 32)])
def test_a_few_short_histories_are_off_by_the_rounding_of_their_results(dtype, d):
    """As above with next to no rows, which smaller workgroups take."""
    dt, H = DT[dtype], 2
    g = torch.Generator(device=DEV).manual_seed(d)
    lens = [1 + (17 * i) % 64 for i in range(60)]
    off, T = ref.offsets(lens), sum(lens)
    q, k, v = (torch.randn(T, H, d, generator=g, device=DEV).to(dt) for _ in range(3))
    out, want = torch.empty_like(q), torch.zeros(T, H, d, dtype=torch.float64, device=DEV)
    hot.dlrm_seq_attn_fwd(hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 64, 64, causal=False), q, k, v, out)
    for s, n in enumerate(lens):
        I = slice(int(off[s]), int(off[s]) + n)
        for h in range(H):
            want[I, h] = torch.softmax(q[I, h].double() @ k[I, h].double().t() * d ** -0.5, -1) @ v[I, h].double()
    err, rounding = norm_off(out, want, dt)
    assert err <= 1.05 * rounding, (err, rounding)


# ------------------------------------------------------------------------------------------------ infinite values
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,B,n", [(64, 3, 40), (64, 200, 64), (64, 40, 200), (128, 30, 152)])
def test_an_infinite_value_is_an_infinite_column_of_who_sees_it(dtype, d, B, n):
    """Every weight is above zero, so the columns are that infinity, and the others finite: sequences of every cut, and the cache."""
    dt, H, page = DT[dtype], 2, 8
    g = torch.Generator(device=DEV).manual_seed(d + n)
    q, k, v = (torch.randn(B * n, H, d, generator=g, device=DEV).to(dt) for _ in range(3))
    v[n // 2::n, :, 3], v[n - 1::n, :, 5] = INF, -INF
    off = torch.arange(B + 1, device=DEV) * n
    out = torch.empty_like(q)
    hot.dlrm_seq_attn_fwd(hot.SeqBatch(off, off, B * n, B * n, n, n, causal=False), q, k, v, out)
    one = q[::n].contiguous()
    pages = lambda x: x.view(B * n // page, page, H, d).transpose(1, 2).contiguous()
    cache = hot.KvCache(pages(k), pages(v), torch.arange(B * n // page, dtype=torch.int32, device=DEV).view(B, -1))
    newest = torch.empty_like(one)
    hot.dlrm_cache_attn(cache, torch.full((B,), n, dtype=torch.int32, device=DEV), n, one, newest, hot.alloc_cache_attn_workspace(cache, H, n))
    cols = torch.ones(d, dtype=torch.bool, device=DEV)
    cols[[3, 5]] = False
    for x in (out, newest):
        assert (x[..., 3] == INF).all() and (x[..., 5] == -INF).all() and torch.isfinite(x[..., cols]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,B,n", [(32, 3, 600), (128, 40, 608), (64, 1, 9000)])
def test_an_infinite_value_in_one_of_several_chunks(dtype, d, B, n):
    """The parts of a long sequence, of attention over sequences and over the cache, are joined to the same infinities."""
    test_an_infinite_value_is_an_infinite_column_of_who_sees_it(dtype, d, B, n)
