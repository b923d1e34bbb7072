"""Attention with a learned bias by buckets in 64 bits, with elementwise error bounds, for the tests.

Bounds as in history_ref: u is the unit roundoff of the storage type, e32 = 2^-24; a score is off by at most e_s (the bias adds its own rounding, 8 e32 |bias|), a
weight by the relative amount 2 e_s + (nk + 16) e32, 16-bit weights and score gradients by u once more in their second product.  The table's gradient sums fp32 score
gradients p (dp - delta): p off by rel_p, dp by (d + 8) e32 |dO| |V|, delta = sum p dp / sum p by what its terms are; and the order of the
sums adds at most their depth times e32 of the sum of magnitudes (a lane adds up to nq terms of a tile's column, then the tiles, then the parts of
all sequences)."""
import math

import torch

from history_ref import E32, TINY, UNIT, visible


def buckets(away, bounds):
    """Number of bounds that are at most each distance, by comparison with every one."""
    b = torch.zeros_like(away)
    for x in ([] if bounds is None else bounds.tolist()):
        b += away >= x
    return b


def scores(q, k, away, slope, bias_row, bounds, scale, cap):
    """(scores, derivative by the product, magnitude that rounding goes by) of one head; away: distances [n, m]."""
    d = q.shape[1]
    x, mag = scale * (q @ k.T), scale * (q.abs() @ k.abs().T)
    t = torch.tanh(x / cap) if cap else torch.zeros_like(x)
    dist = away.abs().double()
    b = torch.zeros_like(x) if bias_row is None else bias_row.double()[buckets(away, bounds)]
    fin = torch.where(b.isinf(), torch.zeros_like(b), b).abs()
    sc = (cap * t if cap else x) - slope * dist
    e = E32 * ((d + 8) * mag + 8 * sc.abs() + 8 * slope * dist + 8 * fin)
    return sc + b, scale * (1 - t * t) if cap else scale * torch.ones_like(x), e


def softmax(sc, seen):
    """(weights, maximum, sum); a row that sees nothing has weights of zero."""
    sc = sc.masked_fill(~seen, -math.inf)
    m = sc.amax(-1, keepdim=True) if sc.shape[-1] else torch.full((sc.shape[0], 1), -math.inf).double()
    any_ = m > -math.inf
    m = torch.where(any_, m, torch.zeros_like(m))
    e = torch.exp(sc - m)
    l = e.sum(-1, keepdim=True)
    return e / torch.where(any_, l, torch.ones_like(l)), m, l, any_


def attention(q, k, v, q_off, k_off, causal, prefix, slopes, table, bounds, scale, cap, dout=None):
    """{"out", "lse", ("dq", "dk", "dv", "dtable")} and the bound of each under "<name>_tol"; all inputs on the host, of the storage type."""
    dt = q.dtype
    u, half = UNIT[dt], dt != torch.float32
    Hq, Hk, d = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hk
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64)
    r = {"out": z(q), "lse": torch.full((Hq, q.shape[0]), -math.inf, dtype=torch.float64), "out_tol": z(q),
         "lse_tol": torch.zeros(Hq, q.shape[0], dtype=torch.float64)}
    if dout is not None:
        r.update({n + t: z(x) for n, x in (("dq", q), ("dk", k), ("dv", v), ("dtable", table)) for t in ("", "_tol")})
    depth = k.shape[0] + len(q_off) + 128
    for s in range(len(q_off) - 1):
        I, J = slice(int(q_off[s]), int(q_off[s + 1])), slice(int(k_off[s]), int(k_off[s + 1]))
        nq, nk = I.stop - I.start, J.stop - J.start
        if not nq or not nk:
            continue
        seen = visible(nq, nk, causal, 0 if prefix is None else int(prefix[s]))
        away = (torch.arange(nq)[:, None] + nk - nq) - torch.arange(nk)[None]
        b = buckets(away, bounds)
        for h in range(Hq):
            Q, K, V = q[I, h].double(), k[J, h // G].double(), v[J, h // G].double()
            sc, slope, e_s = scores(Q, K, away, 0.0 if slopes is None else float(slopes[h]), table[h], bounds, scale, cap)
            e_s = ((e_s + cap * (2.0 ** -20 if half else 2.0 ** -22)) * seen).amax(-1, keepdim=True)
            p, m, l, any_ = softmax(sc, seen)
            rel = 2 * e_s + (nk + 16) * E32
            out, mags = p @ V, p @ V.abs()
            r["out"][I, h], r["out_tol"][I, h] = out, u * out.abs() + (u * half + 2 * rel) * mags + TINY[dt]
            lse = (m + torch.log(torch.where(any_, l, torch.ones_like(l))))[:, 0]
            r["lse"][h, I] = torch.where(any_[:, 0], lse, torch.full_like(lse, -math.inf))
            r["lse_tol"][h, I] = (e_s + (nk + 16) * E32)[:, 0] + 4 * E32 * lse.abs()
            if dout is None:
                continue
            dO = dout[I, h].double()
            dp, delta = dO @ V.T, (dO * out).sum(-1, keepdim=True)
            raw = p * (dp - delta)
            ds = raw * slope
            t_dp = (d + 8) * E32 * (dO.abs() @ V.abs().T)
            off = (dO.abs() * r["out_tol"][I, h]).sum(-1, keepdim=True) + t_dp + (d + 8) * E32 * (dO.abs() * out.abs()).sum(-1, keepdim=True)
            rel_p = rel + e_s + 8 * E32
            bent = p * (dp - delta).abs() * (2.0 ** -19 if half else 2.0 ** -21) if cap else 0.0
            t_ds = u * half * ds.abs() + scale * p * (off + rel_p * (dp.abs() + delta.abs())) + scale * bent
            t_p = (u * half + rel_p) * p
            n_q, n_k = (nk + 16) * E32, (nq * G + 16) * E32
            hk = h // G
            r["dq"][I, h], r["dq_tol"][I, h] = ds @ K, t_ds @ K.abs() + n_q * (ds.abs() @ K.abs()) + TINY[dt]
            r["dk"][J, hk] += ds.T @ Q
            r["dk_tol"][J, hk] += t_ds.T @ Q.abs() + n_k * (ds.T.abs() @ Q.abs()) + TINY[dt]
            r["dv"][J, hk] += p.T @ dO
            r["dv_tol"][J, hk] += t_p.T @ dO.abs() + n_k * (p.T @ dO.abs()) + TINY[dt]
            mean = (p * dp.abs()).sum(-1, keepdim=True)
            t_delta = (p * t_dp).sum(-1, keepdim=True) + (2 * rel_p.clamp(max=1e9) + (nk + 16) * E32) * mean
            t_raw = p * (t_dp + t_delta) + rel_p * p * (dp.abs() + delta.abs()) + (nq + depth) * E32 * raw.abs()
            r["dtable"][h].index_add_(0, b.flatten(), raw.flatten())
            r["dtable_tol"][h].index_add_(0, b.flatten(), t_raw.flatten())
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            r[n + "_tol"] += u * r[n].abs()
        r["dtable_tol"] += 1e-30
    return r


def cached(q, k_old, v_old, k_new, v_new, positions, last, slopes, table, bounds, scale, cap):
    """Attention of one sequence's new items [n, Hq, d] over its cached keys [len, Hk, d] and over one another: (out, bound).  last None: k_new and v_new are
    None too, and the one query stands at the newest cached item."""
    dt = q.dtype
    u, half = UNIT[dt], dt != torch.float32
    n, Hq, d = q.shape
    L, Hk = k_old.shape[:2]
    out, tol = (torch.zeros(n, Hq, d, dtype=torch.float64) for _ in range(2))
    i = torch.arange(n)
    place, seen = torch.arange(L), torch.ones(n, L, dtype=torch.bool)
    if last is not None:
        place = torch.cat([place, positions.long()])
        seen = torch.cat([seen, (i <= i[:, None]) & (i[:, None] <= last.long())], 1)
    away = positions.long()[:, None] - place
    for h in range(Hq):
        hk = h // (Hq // Hk)
        K, V = k_old[:, hk].double(), v_old[:, hk].double()
        if last is not None:
            K, V = torch.cat([K, k_new[:, hk].double()]), torch.cat([V, v_new[:, hk].double()])
        if not K.shape[0]:
            continue
        sc, _, e_s = scores(q[:, h].double(), K, away, 0.0 if slopes is None else float(slopes[h]), None if table is None else table[h], bounds, scale, cap)
        e_s = ((e_s + cap * (2.0 ** -20 if half else 2.0 ** -22)) * seen).amax(-1, keepdim=True)
        p, _, _, _ = softmax(sc, seen)
        rel = 2 * e_s + (K.shape[0] + 16) * E32
        out[:, h] = p @ V
        tol[:, h] = u * out[:, h].abs() + (u * half + 2 * rel) * (p @ V.abs()) + TINY[dt]
    return out, tol
