"""How many digits results with a learned bias have, where the elementwise bounds of bias_ref allow a caller's worst case: results that are only rounded to their
type, and the table's gradient in fp32's digits."""
import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from bias_table_ref import LIMIT, off, table_gradient
from history_ref import offsets
from test_gpu_cache_tree import Paged
from test_gpu_relative_bias import CASES, DEV, DT, gen, rand, run, setup

pytestmark = pytest.mark.gpu


def wrongly_rounded(got, want):
    """Share of the elements that are not the 64-bit value rounded once to their type."""
    return float((got.cpu() != want.to(got.dtype)).double().mean())


@pytest.mark.parametrize("d", [128, 96, 72])
@pytest.mark.parametrize("kind", ["slopes", "bias", "cap"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_queries_gradients_of_wide_rows_are_off_by_their_own_rounding(dtype, kind, d):
    """Slopes and a steep learned bias leave a row few keys of weight.  With up to 32 keys delta is fp32, so what is left is the score gradients' rounding on their way into
    the product.  In two parts that is 2^-17 (bf16) or 2^-22 (fp16) of each, fp32 adds some 2^-20 of a row's magnitudes, and a result that is off by the part x of its spacing
    (2^-8 or 2^-11 of its value, at least) is wrongly rounded in 2x of all cases: about one of 128 in bf16, and a few times that where terms cancel.  In one part score gradients are 2^-9 or
    2^-12 off, a quarter of the spacing at their root mean square: a third of the results.  (The first item of a sequence sees itself alone: its gradient is rounding alone.)"""
    g, dt, Hq, Hk = gen(d), DT[dtype], 4, 2
    lens = [32, 5, 17, 30, 2, 29, 31, 11] * 4
    starts, T = offsets(lens), sum(lens)
    x = {n: rand(g, T, H, d, dtype=dt) for n, H in (("q", Hq), ("k", Hk), ("v", Hk), ("do", Hq))}
    slopes = torch.tensor([0.5, 0.25, 0.7, 0.1]) if kind == "slopes" else None
    bounds = torch.arange(1, 16, dtype=torch.int32)
    table = rand(g, Hq, 16) * (1 if slopes is not None else 2)
    cap = 8.0 if kind == "cap" else 0.0
    seq = hot.SeqBatch(starts.to(DEV), starts.to(DEV), T, T, 32, 32, slopes=None if slopes is None else slopes.to(DEV), cap=cap)
    got = run(x, seq, hot.RelBias(table.to(DEV), bounds.to(DEV)), "rows")
    want = ref.attention(x["q"], x["k"], x["v"], starts, starts, True, None, slopes, table, bounds, d ** -0.5, cap, x["do"])
    more = torch.ones(T, dtype=torch.bool)
    more[starts[:-1]] = False
    share = wrongly_rounded(got["dq"].cpu()[more], want["dq"][more])
    print("[share]", dtype, kind, d, share, flush=True)
    assert share < 0.05


MANY = [
    # query heads, key heads, d, cached, new items, bias, cap
    (4, 2, 64, [300, 17], 3, True, 0.0),          # 6 columns: the kernel for few
    (8, 2, 128, [400, 40], 10, True, 20.0),       # 40: two wavefronts to 32 columns
    (8, 2, 64, [400, 0], 30, False, 0.0),         # 120
    (16, 4, 96, [90, 333], 60, True, 0.0),        # 240: a workgroup of eight wavefronts
    (16, 4, 128, [9000], 64, False, 0.0),         # several chunks
    (8, 1, 40, [1200, 700], 70, True, 30.0),      # several blocks
    (64, 1, 32, [200, 100], 20, False, 0.0),
]


@pytest.mark.parametrize("i", range(len(MANY)))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_new_items_are_off_by_their_own_rounding_however_many(dtype, i):
    """Weights enter their product in two parts, 2^-17 (bf16) or 2^-22 (fp16) of each off: as above, about one result of 128 in bf16 is wrongly rounded, and in one part a third."""
    Hq, Hk, d, lens, m, with_bias, cap = MANY[i]
    g, dt, B = gen(40 + i), DT[dtype], len(lens)
    c = Paged(g, lens, -(-max(lens) // 16), 16, Hk, d, dt)
    x = {n: rand(g, B * m, H, d, dtype=dt) for n, H in (("q", Hq), ("k", Hk), ("v", Hk))}
    pos, last = torch.cat([torch.arange(y, y + m) for y in lens]).to(torch.int32), torch.full((B * m,), m - 1, dtype=torch.int32)
    table, bounds = (rand(g, Hq, 32), hot.relative_bounds(32, 300)) if with_bias else (None, None)
    items = hot.NewItems(offsets([m] * B).to(DEV), B * m, m, positions=pos.to(DEV))
    out = torch.empty_like(x["q"]).to(DEV)
    hot.dlrm_cache_tree_attn(c.cache, c.dlens, max(lens), items, *(x[n].to(DEV) for n in "qkv"), out,
                             hot.alloc_cache_tree_attn_workspace(c.cache, Hq, max(lens), items),
                             bias=hot.RelBias(table.to(DEV), bounds.to(DEV)) if with_bias else None, cap=cap)
    want = torch.cat([ref.cached(x["q"][I], c.k[s], c.v[s], x["k"][I], x["v"][I], pos[I], last[I], None, table, bounds, d ** -0.5, cap)[0]
                      for s, I in ((s, slice(s * m, (s + 1) * m)) for s in range(B))])
    share = wrongly_rounded(out, want)
    print("[share]", dtype, i, share, flush=True)
    assert share < 0.05


@pytest.mark.parametrize("i", range(len(CASES)))
def test_the_table_s_gradient_has_fp32_s_digits(i):
    x, how, seq, bias, where = setup(i)
    got = run(x, seq, bias, where)["dtable"]
    want, size = table_gradient(x, *how)
    print("[off]", i, off(got, want, size), flush=True)
    assert off(got, want, size) < LIMIT


def test_a_cap_beside_a_bias_bends_scores_to_the_last_digits():
    """One key for each query, so lse is the score, cap tanh(z) with a cap of 1.  tanh is off by 2.7e-7 of itself at most (1.02e-7 up to 0.625, by a polynomial), its
    factor log2 e, lse's factor ln 2 and the product of 8 columns by half a step each, with the factors' own roundings 5 half steps of 2^-24."""
    z = torch.cat([torch.logspace(-20, -2, 300, base=2), torch.linspace(0.2, 0.7, 1000), torch.linspace(0.7, 9, 700)])
    z = torch.cat([z, -z])
    T, off_ = z.numel(), torch.arange(z.numel() + 1, device=DEV)
    q, k = torch.zeros(T, 1, 8, device=DEV), torch.zeros(T, 1, 8, device=DEV)
    q[:, 0, 3], k[:, 0, 3] = z.to(DEV), 1.0
    out, lse = torch.empty_like(q), torch.empty(1, T, device=DEV)
    seq = hot.SeqBatch(off_, off_, T, T, 1, 1, scale=1.0, cap=1.0)
    hot.dlrm_seq_attn_bias_fwd(seq, hot.RelBias(torch.zeros(1, 1, device=DEV), None), q, k, k, out, lse)
    want = torch.tanh(z.double())
    off_by = ((lse[0].cpu().double() - want) / want).abs()
    print("[off]", float(off_by[z.abs() <= 0.625].max()), float(off_by[z.abs() > 0.625].max()), flush=True)
    assert bool((off_by <= torch.where(z.abs() <= 0.625, 1.02e-7, 2.7e-7) + 5 * 2.0 ** -24).all())
