"""The table's gradient of a learned bias in 64 bits, with the size that its error is measured by, for the tests; mistakes can be planted in it.

The kernels promise fp32's digits whatever the rows' type.  A pair's score gradient p (dp - delta) is there off by some 10 (1 + |score|) 2^-24 of itself: its product is an fp32 sum
of d terms (sqrt(d)/2 roundings at their root mean square), the score's other steps and the exponential add a few.  These errors have no common sign, so sums over pairs are off by that part of
the root of the sum of their squares: 1e-6 to 2e-6 of it for scores of ordinary size, and LIMIT is five times the larger.  An operand of 16 bits in place of one of 32 makes it 2^-9 or
2^-12."""
import math

import torch

from bias_ref import buckets, softmax
from history_ref import visible

LIMIT = 1e-5


def table_gradient(x, q_off, k_off, causal, prefix, slopes, table, bounds, scale, cap, mistake=None):
    """(gradient [Hq, n], root of the sum of the squares of the pairs' score gradients)"""
    dt = x["q"].dtype
    Hq, Hk = x["q"].shape[1], x["k"].shape[1]
    grad, squares = torch.zeros(table.shape, dtype=torch.float64), 0.0
    narrow = lambda y: y.to(dt).double()
    for s in range(len(q_off) - 1):
        I, J = slice(int(q_off[s]), int(q_off[s + 1])), slice(int(k_off[s]), int(k_off[s + 1]))
        nq, nk = I.stop - I.start, J.stop - J.start
        if not nq or not nk:
            continue
        seen = visible(nq, nk, causal, 0 if prefix is None else int(prefix[s]))
        away = (torch.arange(nq)[:, None] + nk - nq) - torch.arange(nk)[None]
        b = buckets(away, bounds)
        for h in range(Hq):
            hk = h // (Hq // Hk)
            Q, K, V, D = (x[n][R, i].double() for n, R, i in (("q", I, h), ("k", J, hk), ("v", J, hk), ("do", I, h)))
            sc = scale * (Q @ K.T)
            sc = cap * torch.tanh(sc / cap) if cap else sc
            sc = sc + table[h].double()[b] - (0.0 if slopes is None else float(slopes[h])) * away.abs().double()
            p = softmax(sc, seen)[0]
            dp = D @ V.T
            delta = (p * dp).sum(-1, keepdim=True)
            if mistake == "weights":
                p = narrow(p)
            if mistake == "delta":
                delta = (narrow(p @ V) * D).sum(-1, keepdim=True)
            ds = p * (dp - delta)
            if mistake == "score gradients":
                ds = narrow(ds)
            grad[h].index_add_(0, b.flatten(), ds.flatten())
            squares += float(ds.square().sum())
    return grad, math.sqrt(squares)


def off(got, want, size):
    return float((got.double().cpu() - want).norm()) / size
