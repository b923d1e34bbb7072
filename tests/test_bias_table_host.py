"""That the limit on the table's gradient (bias_table_ref) tells fp32's digits from those of a narrower operand: mistakes planted in the 64-bit form."""
import pytest
import torch

import paper_1906_00091_amd as hot

import bias_ref as ref
from bias_table_ref import LIMIT, off, table_gradient
from history_ref import offsets

CASES = [  # type, query heads, key heads, d, lengths, causal, slopes, cap, buckets
    (torch.bfloat16, 8, 2, 128, [90, 300], True, False, 20.0, 20),
    (torch.bfloat16, 4, 2, 128, [260, 40], True, False, 30.0, 64),
    (torch.bfloat16, 4, 4, 64, [200, 1, 0, 77], True, False, 0.0, 32),
    (torch.bfloat16, 2, 1, 96, [150, 80], False, True, 0.0, 17),
    (torch.float16, 4, 2, 128, [200, 130], True, False, 10.0, 31),
    (torch.float16, 2, 2, 40, [250, 30], False, False, 0.0, 33),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_narrow_operands_pass_the_limit(i):
    dt, Hq, Hk, d, lens, causal, slopes, cap, n = CASES[i]
    g, o, T = torch.Generator().manual_seed(i), offsets(lens), sum(lens)
    x = {name: torch.randn(T, H, d, generator=g).to(dt) for name, H in (("q", Hq), ("k", Hk), ("v", Hk), ("do", Hq))}
    how = (o, o, causal, None, torch.rand(Hq, generator=g) * 0.2 if slopes else None, torch.randn(Hq, n, generator=g), hot.relative_bounds(n, 100, not causal),
           d ** -0.5, cap)
    want, size = table_gradient(x, *how)
    assert off(ref.attention(x["q"], x["k"], x["v"], *how, dout=x["do"])["dtable"], want, size) < 1e-12   # the same as the elementwise form's
    assert size < 10 * float(want.norm())   # (the limit means what it says of the gradient itself)
    for mistake in ("weights", "delta", "score gradients"):
        wrong = table_gradient(x, *how, mistake=mistake)[0]
        print("[off]", i, mistake, off(wrong, want, size))
        assert off(wrong, want, size) > 4 * LIMIT, mistake
