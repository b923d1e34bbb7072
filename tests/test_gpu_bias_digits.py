"""How many digits results with a learned bias have, where the elementwise bounds of bias_ref allow a caller's worst case: results that are only rounded to their
type, and the table's gradient in fp32's digits."""
import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from history_ref import offsets
from test_gpu_relative_bias import DEV, DT, gen, rand, run

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
    off, T = offsets(lens), sum(lens)
    x = {n: rand(g, T, H, d, dtype=dt) for n, H in (("q", Hq), ("k", Hk), ("v", Hk), ("do", Hq))}
    slopes = torch.tensor([0.5, 0.25, 0.7, 0.1]) if kind == "slopes" else None
    bounds = torch.arange(1, 16, dtype=torch.int32)
    table = rand(g, Hq, 16) * (1 if slopes is not None else 2)
    cap = 8.0 if kind == "cap" else 0.0
    seq = hot.SeqBatch(off.to(DEV), off.to(DEV), T, T, 32, 32, slopes=None if slopes is None else slopes.to(DEV), cap=cap)
    got = run(x, seq, hot.RelBias(table.to(DEV), bounds.to(DEV)), "rows")
    want = ref.attention(x["q"], x["k"], x["v"], off, off, True, None, slopes, table, bounds, d ** -0.5, cap, x["do"])
    more = torch.ones(T, dtype=torch.bool)
    more[off[:-1]] = False
    share = wrongly_rounded(got["dq"].cpu()[more], want["dq"][more])
    print("[share]", dtype, kind, d, share, flush=True)
    assert share < 0.05
