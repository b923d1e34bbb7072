"""fp16 rows whose weights or gradients leave the exponents that fp16 has at full precision (2^-14 to 2^15): many keys, small and large upstream
gradients.  U = 2^-11 is the unit roundoff; what a number below 2^-14 loses is absolute, 2^-25."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -11
H16 = torch.float16


def attend(q, k, v, do, scale, causal, cap=0.0, slopes=None):
    """The operators' results and those of the formula in 64 bits on the device; one head, one sequence."""
    nq, nk, d = q.shape[0], k.shape[0], q.shape[1]
    Q, K, V, DO = (x.to(H16)[:, None].contiguous() for x in (q, k, v, do))
    seq = hot.SeqBatch(torch.tensor([0, nq], device=DEV), torch.tensor([0, nk], device=DEV), nq, nk, nq, nk, causal=causal, scale=scale, cap=cap,
                       slopes=None if slopes is None else torch.tensor([slopes], device=DEV))
    out, dq, dk, dv = (torch.empty_like(x) for x in (Q, Q, K, V))
    lse = torch.empty(1, nq, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, Q, K, V, out, lse)
    hot.dlrm_seq_attn_bwd(seq, Q, K, V, out, lse, DO, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, 1, 1, d))
    q, k, v, do = (x[:, 0].double() for x in (Q, K, V, DO))
    x = scale * (q @ k.t())
    f = torch.full_like(x, scale)
    if cap:
        t = torch.tanh(x / cap)
        x, f = cap * t, scale * (1 - t * t)
    at = torch.arange(nq, device=DEV)[:, None] + nk - nq - torch.arange(nk, device=DEV)
    if slopes is not None:
        x = x - slopes * at.abs()
    if causal:
        x = x.masked_fill(at < 0, -math.inf)
    p = torch.softmax(x, -1)
    o = p @ v
    ds = p * (do @ v.t() - (do * o).sum(-1, keepdim=True)) * f
    want = {"out": o, "dq": ds @ k, "dk": ds.t() @ q, "dv": p.t() @ do}
    return {n: y[:, 0] for n, y in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv))}, want


def off_by(got, want):
    """Distance from `want` in the Euclidean norm, and how far the nearest fp16 numbers are, both relative to it."""
    size = want.norm()
    return float((got.double() - want).norm() / size), float((want.to(H16).double() - want).norm() / size)


CASES = [
    # d, keys, causal, cap, slopes
    (64, 2048, True, 0.0, None),
    (128, 2048, True, 30.0, None),
    (32, 3000, False, 0.0, 2.0 ** -8),
    (128, 2100, False, 0.0, None),
]


@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4, 1e3])
@pytest.mark.parametrize("d,n,causal,cap,slopes", CASES)
def test_gradients_of_small_and_large_upstream_gradients(d, n, causal, cap, slopes, size):
    """Weights, ds and the result are each rounded once, to a relative U at most, independently: together they move a gradient by less than 2 U of its norm
    (three errors of U / sqrt(3) at most in the mean square, as many again left for delta and fp32), beside the result's own rounding
    where that is below fp16's full precision.  Keys, or queries, of size 2^-6 under a scale 2^6 times as large keep the other's gradient well above that."""
    for small in "kq":
        g = torch.Generator(device=DEV).manual_seed(d + n)
        q, k, v, do = (torch.randn(n, d, generator=g, device=DEV) for _ in range(4))
        q, k = (q, k / 64) if small == "k" else (q / 64, k)
        got, want = attend(q, k, v / (64 if size > 1 else 1), do * size, 64 * d ** -0.5, causal, cap, slopes)
        for name in ("dk", "dv") if small == "k" else ("dq",):
            assert torch.isfinite(got[name]).all(), (name, size)
            err, nearest = off_by(got[name], want[name])
            assert err <= 2 * U + nearest, (name, small, err, nearest)


@pytest.mark.parametrize("d", [40, 128])
def test_score_gradients_beyond_fp16(d):
    """dp - delta of some 10^5, ds with it where few keys share a row; scaled down, dq and dk are ordinary numbers."""
    g = torch.Generator(device=DEV).manual_seed(d)
    n = 300
    q, k, v, do = (torch.randn(n, d, generator=g, device=DEV) for _ in range(4))
    got, want = attend(q, k, v * 16, do * 2000, 2.0 ** -10, True)
    assert float((do.to(H16).double() * 1).abs().max()) > 0 and float(want["dq"].abs().max()) < 30000
    ds = torch.full((), float((do.double() * 2000).norm(dim=-1).max() * (v.double() * 16).norm(dim=-1).max()))
    assert float(ds) > 65504
    for name in ("dq", "dk", "dv"):
        assert torch.isfinite(got[name]).all(), name
        err, nearest = off_by(got[name], want[name])
        assert err <= 2 * U + nearest, (name, err, nearest)


def test_weights_far_below_the_largest_still_sum():
    """One key of weight 1 and value 0, thousands of weight 2^-26 and value 1000.  A weight is held to 2^-25 of 2^-7 of the largest: n 2^-32 |v| in all."""
    n, d = 4096, 16
    q, k, v = (torch.zeros(n if i else 1, d, device=DEV) for i in range(3))
    q[0, 0], k[0, 0], v[1:] = 1.0, 26 * math.log(2.0), 1000.0
    got, want = attend(q, k, v, torch.ones(1, d, device=DEV), 1.0, True)
    assert float((got["out"].double() - want["out"]).abs().max()) <= 4 * U * float(want["out"].max()) + n * 2.0 ** -32 * 1000


def test_cached_weights_far_below_the_largest_still_sum():
    """The same over the cache, where no weight is above 1 and 2^15 times as much is held: n 2^-40 |v| in all."""
    n, d, page, B = 4096, 16, 512, 1024
    k, v = (torch.zeros(n // page, 1, page, d, dtype=H16, device=DEV) for _ in range(2))
    k[0, 0, 0, 0], v[:] = 26 * math.log(2.0), 1000.0
    v[0, 0, 0] = 0.0
    q = torch.zeros(B, 1, d, dtype=H16, device=DEV)
    q[:, 0, 0] = 1.0
    cache = hot.KvCache(k, v, torch.arange(n // page, dtype=torch.int32, device=DEV).repeat(B, 1))
    out = torch.empty_like(q)
    hot.dlrm_cache_attn(cache, torch.full((B,), n, dtype=torch.int32, device=DEV), n, q, out, hot.alloc_cache_attn_workspace(cache, 1, n), scale=1.0)
    w = math.exp(float(k[0, 0, 0, 0]))
    want = 1000.0 * (n - 1) / (n - 1 + w)
    assert float((out.double() - want).abs().max()) <= 4 * U * want + n * 2.0 ** -40 * 1000


def test_equal_weights_of_very_many_keys():
    """p = 100.5 units of 2^-24 for every key: dv is the number of queries times it."""
    nq, nk, d = 64, 166936, 8
    q, k, v = torch.zeros(nq, d, device=DEV), torch.zeros(nk, d, device=DEV), torch.ones(nk, d, device=DEV)
    n1 = torch.ones(nq, d, device=DEV)
    got, want = attend(q, k, v, n1, 1.0, False)
    assert float((got["dv"].double() / want["dv"] - 1).abs().max()) <= 2 * U
    assert float((got["out"].double() - 1).abs().max()) <= 2 * U
