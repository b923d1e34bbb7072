"""Attention over sequences with scores that are all zero, so that results are counts: every visible key, or query, once.  Each sum has terms of one sign
in each column (rows are unit vectors e(i mod d)), a column has n / d of them, and one too few or too many moves it by d / n of itself at
least, while it is rounded to 2 or 3 u."""
import math

import pytest
import torch

import paper_1906_00091_amd as hot

import history_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

CASES = [
    # type, d, query heads, key heads, lengths, causal, prefix; enough or few enough rows for each cut of the kernels
    ("f32", 16, 2, 2, [40, 0, 33, 64] * 30, True, False),
    ("f32", 64, 2, 1, [2, 700], True, False),
    ("f32", 32, 4, 4, [200, 130, 1] * 25, True, True),
    ("f32", 24, 32, 32, [2100, 60], True, False),
    ("f32", 96, 4, 4, [257, 90], False, False),
    ("bf16", 16, 8, 2, [64, 0, 33, 20] * 300, True, False),
    ("bf16", 64, 4, 4, [200, 130, 1, 65] * 30, True, False),
    ("f16", 64, 4, 1, [200, 130, 1, 65] * 30, True, True),
    ("bf16", 128, 16, 4, [600, 333] * 6, True, False),
    ("f16", 96, 12, 12, [500, 700] * 8, True, True),
    ("bf16", 32, 4, 2, [600, 20], True, False),
    ("bf16", 128, 2, 2, [1023], False, False),
    ("f16", 16, 1, 1, [5, 700], True, False),
]


def unit_rows(T, H, d, dt):
    x = torch.zeros(T, H, d, dtype=dt)
    x[torch.arange(T), :, torch.arange(T) % d] = 1
    return x


@pytest.mark.parametrize("i", range(len(CASES)))
def test_every_visible_key_and_query_counts_once(i):
    print("[case]", i, CASES[i], flush=True)
    dtype, d, Hq, Hk, lens, causal, prefix = CASES[i]
    dt, off, T = DT[dtype], ref.offsets(lens), sum(lens)
    pre = torch.tensor([n // 4 for n in lens], dtype=torch.int32) if prefix else None
    od = off.to(DEV)
    seq = hot.SeqBatch(od, od, T, T, max(lens), max(lens), causal=causal, prefix=None if pre is None else pre.to(DEV), scale=1.0)
    q1, k1 = unit_rows(T, Hq, d, dt), unit_rows(T, Hk, d, dt)
    sign = torch.zeros(T, Hk, d, dtype=dt)
    sign[..., 0] = (1 - 2 * (torch.arange(T) % 2))[:, None].to(dt)
    first = torch.zeros(T, Hq, d, dtype=dt)
    first[..., 0] = 1

    def run(q, k, v, do):
        q, k, v, do = (x.to(DEV) for x in (q, k, v, do))
        out, dq, dk, dv = (torch.full_like(x, math.nan) for x in (q, q, k, v))
        lse = torch.empty(Hq, T, device=DEV)
        hot.dlrm_seq_attn_fwd(seq, q, k, v, out, lse)
        hot.dlrm_seq_attn_bwd(seq, q, k, v, out, lse, do, dq, dk, dv, hot.alloc_seq_attn_workspace(seq, Hq, Hk, d))
        return {n: x.double().cpu() for n, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv))}
    counts = run(torch.zeros_like(q1), k1, k1, q1)                   # out: keys of a column; dv: queries of a column
    dq = run(torch.zeros_like(q1), k1, sign, first)["dq"]           # ds = (+-1 - delta) / n, its sign that of the key's place
    dk = run(q1, torch.zeros_like(k1), sign, first)["dk"]
    tol = 3 * ref.UNIT[dt] + 2.0 ** -18                             # 2^-18: lse and the weight's exponential in fp32
    for s, n in enumerate(lens):
        if not n:
            continue
        I = slice(int(off[s]), int(off[s]) + n)
        p = ref.visible(n, n, causal, 0 if pre is None else int(pre[s])).double()
        p /= p.sum(-1, keepdim=True)
        e, f, sg = q1[I, 0].double(), k1[I, 0].double(), sign[I, 0, :1].double()
        ds = p * (sg.t() - p @ sg)
        for name, got, want in (("out", counts["out"], p @ f), ("dv", counts["dv"], Hq // Hk * (p.t() @ e)), ("dq", dq, ds @ f),
                                ("dk", dk, Hq // Hk * (ds.t() @ e))):
            bound = tol * want.abs()
            if name in ("dq", "dk"):                                # ds loses delta / (1 - delta) of that again, and 2^-25 below fp16's full precision
                bound = 2 * bound + (2.0 ** -25 if dt == torch.float16 else 0.0)
            bad = ~((got[I] - want[:, None]).abs() <= bound[:, None])
            assert not bad.any(), (name, s, n, torch.nonzero(bad)[0].tolist(), float(got[I][bad][0]), float(want[:, None].expand_as(bad)[bad][0]))
