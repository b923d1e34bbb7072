"""Plain 64-bit forms of the operators that read a history in order, with elementwise error bounds, for the tests.

Bounds: u is the unit roundoff of the storage type (2^-p for p significant bits: 2^-24, 2^-11, 2^-8), e32 = 2^-24.  Each stored value is rounded
once (u |y|).  With 16-bit types weights p and score gradients ds are rounded before their second product (u times
the product of the magnitudes).  What fp32 arithmetic adds: a score is off by at most e_s = e32 ((d + 8) scale sum |q||k| + 8 |score| +
8 slope distance) + cap * 2^-20 (16-bit: one exponential and one reciprocal, each good to 2^-22) or cap * 2^-22, so a weight by the
relative amount 2 e_s, its sum over n keys by n e32 more."""
import math

import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-30, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-30}   # spacing below the normal range
E32 = 2.0 ** -24


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int64)


def rope(x, w, positions, inv_freq, rot, layout, eps, mscale, sign=1.0):
    """y of one [T, H, d] set of rows, in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    return turn(x, positions, inv_freq, rot, layout, mscale, sign)


def turn(x, positions, inv_freq, rot, layout, mscale, sign=1.0):
    if not rot:
        return x
    a = positions.double()[:, None, None] * inv_freq.double()
    c, s = mscale * a.cos(), mscale * sign * a.sin()
    y = x.clone()
    at = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    p, q = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = p * c - q * s, q * c + p * s
    return y


def rope_grad(x, w, dy, positions, inv_freq, rot, layout, eps, mscale):
    """(dx, dw) by the chain rule, in 64 bits."""
    x, g = x.double(), turn(dy.double(), positions, inv_freq, rot, layout, mscale, -1.0)
    if w is None:
        return g, None
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n, gw = x * r, g * w.double()
    return r * (gw - n * (gw * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def visible(nq, nk, causal, prefix):
    p = torch.arange(nq)[:, None] + (nk - nq)
    j = torch.arange(nk)[None]
    return (j <= p) | (j < prefix) if causal else torch.ones(nq, nk, dtype=torch.bool)


def attention(q, k, v, q_off, k_off, causal, prefix, slopes, scale, cap, dout=None):
    """{"out", "lse", ("dq", "dk", "dv")} and the bound of each under "<name>_tol"; all inputs on the host, of the storage type."""
    dt = q.dtype
    u, half = UNIT[dt], dt != torch.float32
    Hq, Hk, d = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hk
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64)
    r = {"out": z(q), "lse": torch.full((Hq, q.shape[0]), -math.inf, dtype=torch.float64), "out_tol": z(q),
         "lse_tol": torch.zeros(Hq, q.shape[0], dtype=torch.float64)}
    if dout is not None:
        r.update({n + t: z(x) for n, x in (("dq", q), ("dk", k), ("dv", v)) for t in ("", "_tol")})
    for s in range(len(q_off) - 1):
        I, J = slice(int(q_off[s]), int(q_off[s + 1])), slice(int(k_off[s]), int(k_off[s + 1]))
        nq, nk = I.stop - I.start, J.stop - J.start
        if not nq or not nk:
            continue
        seen = visible(nq, nk, causal, 0 if prefix is None else int(prefix[s]))
        dist = ((torch.arange(nq)[:, None] + nk - nq) - torch.arange(nk)[None]).abs().double()
        for h in range(Hq):
            Q, K, V = q[I, h].double(), k[J, h // G].double(), v[J, h // G].double()
            x, mag = scale * (Q @ K.T), scale * (Q.abs() @ K.abs().T)
            t = torch.tanh(x / cap) if cap else torch.zeros_like(x)
            sl = 0.0 if slopes is None else float(slopes[h])
            sc = (cap * t if cap else x) - sl * dist
            e_s = E32 * ((d + 8) * mag + 8 * sc.abs() + 8 * sl * dist) + cap * (2.0 ** -20 if half else 2.0 ** -22)
            e_s = (e_s * seen).amax(-1, keepdim=True)
            sc = sc.masked_fill(~seen, -math.inf)
            any_ = seen.any(-1, keepdim=True)
            m = torch.where(any_, sc.amax(-1, keepdim=True), torch.zeros(()).double())
            e = torch.exp(sc - m)
            l = e.sum(-1, keepdim=True)
            p = e / torch.where(any_, l, torch.ones_like(l))
            rel = 2 * e_s + (nk + 16) * E32              # of a weight, from fp32 arithmetic
            out, mags = p @ V, p @ V.abs()
            r["out"][I, h], r["out_tol"][I, h] = out, u * out.abs() + (u * half + 2 * rel) * mags + TINY[dt]
            lse = (m + torch.log(torch.where(any_, l, torch.ones_like(l))))[:, 0]
            r["lse"][h, I] = torch.where(any_[:, 0], lse, torch.full_like(lse, -math.inf))
            r["lse_tol"][h, I] = (e_s + (nk + 16) * E32)[:, 0] + 4 * E32 * lse.abs()
            if dout is None:
                continue
            dO = dout[I, h].double()
            dp, delta = dO @ V.T, (dO * out).sum(-1, keepdim=True)
            f = scale * (1 - t * t) if cap else scale * torch.ones_like(x)
            ds = p * (dp - delta) * f
            # delta comes from the stored output; both products are fp32 sums of d terms
            off = (dO.abs() * r["out_tol"][I, h]).sum(-1, keepdim=True) + (d + 8) * E32 * (dO.abs() @ V.abs().T + (dO.abs() * out.abs()).sum(-1, keepdim=True))
            rel_p = rel + e_s + 8 * E32
            t_ds = u * half * ds.abs() + scale * p * (off + rel_p * (dp.abs() + delta.abs())) + (scale * p * (dp - delta).abs() * (2.0 ** -19 if half else 2.0 ** -21) if cap else 0)
            t_p = (u * half + rel_p) * p
            n_q, n_k = (nk + 16) * E32, (nq * G + 16) * E32   # fp32 accumulation
            hk = h // G
            r["dq"][I, h], r["dq_tol"][I, h] = ds @ K, t_ds @ K.abs() + n_q * (ds.abs() @ K.abs()) + TINY[dt]
            r["dk"][J, hk] += ds.T @ Q
            r["dk_tol"][J, hk] += t_ds.T @ Q.abs() + n_k * (ds.T.abs() @ Q.abs()) + TINY[dt]
            r["dv"][J, hk] += p.T @ dO
            r["dv_tol"][J, hk] += t_p.T @ dO.abs() + n_k * (p.T @ dO.abs()) + TINY[dt]
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            r[n + "_tol"] += u * r[n].abs()
    return r


def close(got, want, tol, what):
    """Elementwise: |got - want| <= tol, and the same infinities."""
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = got == want
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    bad = ~(off <= tol) & ~same
    if bad.any():
        i = int(torch.nonzero(bad.flatten())[0])
        raise AssertionError("%s: %d of %d off; first at %d: %r for %r, allowed %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(got.flatten()[i]), float(want.flatten()[i]), float(tol.expand_as(want).flatten()[i])))
