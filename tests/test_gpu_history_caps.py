"""Caps of any size on the scores of 16-bit rows: the score's error must not grow with the cap.  lse, which is fp32, shows it; what the rest may be off by
is u = 2^-11 or 2^-8 a rounding."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def formula(q, k, v, do, scale, cap, slope, causal):
    """One head and sequence in 64 bits."""
    nq, nk = q.shape[0], k.shape[0]
    x = scale * (q @ k.t())
    t = torch.tanh(x / cap)
    away = torch.arange(nq, device=DEV)[:, None] + nk - nq - torch.arange(nk, device=DEV)
    x = cap * t - slope * away.abs()
    if causal:
        x = x.masked_fill(away < 0, -math.inf)
    p = torch.softmax(x, -1)
    o = p @ v
    ds = p * (do @ v.t() - (do * o).sum(-1, keepdim=True)) * scale * (1 - t * t)
    return {"out": o, "lse": torch.logsumexp(x, -1), "dq": ds @ k, "dk": ds.t() @ q, "dv": p.t() @ do}


@pytest.mark.parametrize("cap", [20.0, 129.0, 1000.0, 1025.0, 1e5, 1e9])
@pytest.mark.parametrize("dtype,d,nq,nk,causal,slope", [("f16", 64, 300, 300, True, 0.0), ("bf16", 128, 40, 700, True, 0.125), ("bf16", 32, 33, 20, False, 0.0),
                                                       ("f16", 96, 700, 700, True, 0.0)])
def test_scores_under_caps_of_any_size(dtype, d, nq, nk, causal, slope, cap):
    g, dt, u = torch.Generator(device=DEV).manual_seed(d), DT[dtype], ref.UNIT[DT[dtype]]
    q, do = (torch.randn(nq, 2, d, generator=g, device=DEV).to(dt) for _ in range(2))
    k, v = (torch.randn(nk, 2, d, generator=g, device=DEV).to(dt) for _ in range(2))
    sl = torch.tensor([slope, slope / 2], device=DEV) if slope else None
    scale = 2 * d ** -0.5
    seq = hot.SeqBatch(torch.tensor([0, nq], device=DEV), torch.tensor([0, nk], device=DEV), nq, nk, nq, nk, causal=causal, scale=scale, cap=cap, slopes=sl)
    out, dq, dk, dv = (torch.empty_like(x) for x in (q, q, k, v))
    lse = torch.empty(2, nq, device=DEV)
    hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
    hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, 2, 2, d))
    got = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    for h in range(2):
        want = formula(*(x[:, h].double() for x in (q, k, v, do)), scale, cap, 0.0 if sl is None else float(sl[h]), causal)
        # a score: the fp32 product's (d + 8) 2^-24 of its magnitude, below 2 d; a cap that is taken the short way 2^-21 of it, at most u / 8; 2^-20 for the rest
        e = (d + 8) * 2.0 ** -24 * 2 * d + min(cap * 2.0 ** -21, u / 8) + 2.0 ** -20
        assert float((lse[h].double() - want["lse"]).abs().max()) <= e
        for n, x in got.items():
            err = float((x[:, h].double() - want[n]).norm() / want[n].norm())
            assert err <= 2 * u, (n, h, err)


@pytest.mark.parametrize("cap", [20.0, 1000.0, 1e5, 1e9])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_cached_scores_under_caps_of_any_size(dtype, cap):
    g, dt, B, H, d, page, n = torch.Generator(device=DEV).manual_seed(3), DT[dtype], 3, 4, 64, 32, 640
    q = torch.randn(B, H, d, generator=g, device=DEV).to(dt)
    k, v = (torch.randn(B * n // page, H, page, d, generator=g, device=DEV).to(dt) for _ in range(2))
    cache = hot.KvCache(k, v, torch.arange(B * n // page, dtype=torch.int32, device=DEV).view(B, -1))
    out = torch.empty_like(q)
    hot.dlrm_cache_attn(cache, torch.full((B,), n, dtype=torch.int32, device=DEV), n, q, out, hot.alloc_cache_attn_workspace(cache, H, n), scale=2 * d ** -0.5, cap=cap)
    K, V = (x.double().view(B, n // page, H, page, d).transpose(2, 3).reshape(B, n, H, d) for x in (k, v))
    for b in range(B):
        for h in range(H):
            want = formula(q[b, h:h + 1].double(), K[b, :, h], V[b, :, h], q[b, h:h + 1].double(), 2 * d ** -0.5, cap, 0.0, False)["out"]
            assert float((out[b, h:h + 1].double() - want).norm() / want.norm()) <= 2 * ref.UNIT[dt]
