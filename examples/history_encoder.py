"""A sequence encoder between the row lookup and the scores: a user's history of items, read in order.

    python examples/history_encoder.py [--steps 30] [--users 256] [--items 20000] [--seed 1]

Training: the rows of a history's items are looked up (dlrm_emb_bag_fwd, one index a bag), projected to queries, keys and values, normed and
rotated (dlrm_qk_rope_fwd), attended causally within each history (dlrm_seq_attn_fwd), and projected back beside the rows themselves.  The
vector of every item but the last scores the item that follows it against a random one (logistic loss).  The gradients go back the same way
(dlrm_seq_attn_bwd, dlrm_qk_rope_bwd) and into the table's rows (dlrm_emb_bag_bwd_sgd).  Projections are torch products.

Serving: the histories go into a paged cache (dlrm_qk_rope_append), then every user's newest item alone is run against it
(dlrm_qk_rope_append, dlrm_cache_attn) and compared with the whole history run at once."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1906_00091_amd as hot  # noqa: E402

DEV = "cuda:0"


class Encoder:
    def __init__(self, items, width=64, Hq=4, Hk=2, d=32, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        w = lambda *s: torch.randn(*s, generator=g, device=DEV) * s[0] ** -0.5
        self.Hq, self.Hk, self.d, self.width = Hq, Hk, d, width
        self.table = torch.empty(items, width, device=DEV)
        hot.dlrm_table_init_hash(self.table, hot.F32, seed, 0.3)
        self.qkv, self.back = w(width, (Hq + 2 * Hk) * d), w(Hq * d, width)
        self.wq, self.wk = torch.ones(d, device=DEV), torch.ones(d, device=DEV)
        self.freq = hot.rope_frequencies(d, device=DEV)

    def lookup(self, items):
        """Rows of items [T], and the batch they were looked up with."""
        T = items.numel()
        offsets = torch.arange(T + 1, device=DEV).view(1, -1)
        batch = hot.SparseBatch([self.table], hot.F32, items, offsets, torch.tensor([0, T], device=DEV), T)
        x = torch.empty(T, 1, self.width, device=DEV)
        hot.dlrm_emb_bag_fwd(batch, x, self.width, self.width)
        return x.view(T, self.width), batch

    def project(self, x):
        p = (x @ self.qkv).view(x.shape[0], self.Hq + 2 * self.Hk, self.d)
        return p, p[:, :self.Hq], p[:, self.Hq:self.Hq + self.Hk], p[:, self.Hq + self.Hk:]

    def rope(self, positions):
        return hot.QkRope(positions, self.Hq, self.Hk, self.d, inv_freq=self.freq, wq=self.wq, wk=self.wk)


def histories(lengths):
    """(offsets on the device, position of every item, user of every item, the attention's batch)"""
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)])).to(DEV)
    users = torch.from_numpy(np.repeat(np.arange(len(lengths)), lengths)).to(DEV)
    T = int(sum(lengths))
    positions = (torch.arange(T, device=DEV) - off[users]).to(torch.int32)
    top = int(max(lengths))
    return off, positions, users.to(torch.int32), hot.SeqBatch(off, off, T, T, top, top)


def encode(m, x, positions, seq):
    """Vectors [T, width] of all items and what the way back needs."""
    T = x.shape[0]
    rope = m.rope(positions)
    p, q, k, v = m.project(x)
    qr, kr, o = (torch.empty(T, H, m.d, device=DEV) for H in (m.Hq, m.Hk, m.Hq))
    lse = torch.empty(m.Hq, T, device=DEV)
    hot.dlrm_qk_rope_fwd(rope, q, k, qr, kr)
    hot.dlrm_seq_attn_fwd(seq, qr, kr, v, o, lse)
    return x + o.view(T, -1) @ m.back, (rope, p, q, k, v, qr, kr, o, lse)


def train_step(m, lengths, items, others, lr, row_lr):
    """One step on histories of the given lengths; items: [T]; others: [T] random items; row_lr: the table's, whose rows each see
    a few of the batch's items only.  Returns the mean loss."""
    T = items.numel()
    off, positions, _, seq = histories(lengths)
    x, batch = m.lookup(items)
    y, _ = m.lookup(others)
    u, (rope, p, q, k, v, qr, kr, o, lse) = encode(m, x, positions, seq)
    last = torch.zeros(T, dtype=torch.bool, device=DEV)
    last[off[1:] - 1] = True
    n = T - int(last.sum())
    following = torch.roll(x, -1, 0)
    good, bad = (u * following).sum(-1), (u * y).sum(-1)
    loss = torch.nn.functional.softplus(-good) + torch.nn.functional.softplus(bad)
    loss = loss.masked_fill(last, 0).sum() / n
    # the way back
    ggood = (-torch.sigmoid(-good)).masked_fill(last, 0)[:, None] / n
    gbad = torch.sigmoid(bad).masked_fill(last, 0)[:, None] / n
    du = ggood * following + gbad * y
    dx = du + torch.roll(ggood * u, 1, 0)
    do = (du @ m.back.t()).view(T, m.Hq, m.d)
    dp = torch.empty_like(p)
    dq, dk, dv = dp[:, :m.Hq], dp[:, m.Hq:m.Hq + m.Hk], dp[:, m.Hq + m.Hk:]
    dqr, dkr = torch.empty_like(qr), torch.empty_like(kr)
    hot.dlrm_seq_attn_bwd(seq, qr, kr, v, o, lse, do, dqr, dkr, dv, hot.alloc_seq_attn_workspace(seq, m.Hq, m.Hk, m.d))
    dw = torch.empty(2, m.d, device=DEV)
    hot.dlrm_qk_rope_bwd(rope, q, k, dqr, dkr, dq, dk, dw[0], dw[1], hot.alloc_qk_rope_workspace(rope))
    dp = dp.view(T, -1)
    dx = (dx + dp @ m.qkv.t()).contiguous()
    for w, g in ((m.back, o.view(T, -1).t() @ du), (m.qkv, x.t() @ dp), (m.wq, dw[0]), (m.wk, dw[1])):
        w.sub_(lr * g)
    hot.dlrm_emb_bag_bwd_sgd(batch, dx, m.width, m.width, row_lr, hot.alloc_workspace(batch))
    return float(loss)


def serve(m, lengths, items, page=16):
    """Every history into the cache but for its newest item, that item alone against the cache; returns the vectors of the newest items
    and those of the whole histories run at once."""
    off, positions, users, seq = histories(lengths)
    x, _ = m.lookup(items)
    whole, _ = encode(m, x, positions, seq)
    newest = off[1:] - 1
    old = torch.ones(items.numel(), dtype=torch.bool, device=DEV)
    old[newest] = False
    B, cols = len(lengths), (max(lengths) + page - 1) // page
    pool = torch.empty(2, B * cols, m.Hk, page, m.d, device=DEV)
    cache = hot.KvCache(pool[0], pool[1], torch.randperm(B * cols, device=DEV).to(torch.int32).view(B, cols))
    for now in (old, ~old):
        at = positions[now].contiguous()
        _, q, k, v = m.project(x[now])
        qr = torch.empty(at.numel(), m.Hq, m.d, device=DEV)
        hot.dlrm_qk_rope_append(m.rope(at), q, k, v, qr, cache, users[now].contiguous())
    o = torch.empty_like(qr)
    top = max(lengths)
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    hot.dlrm_cache_attn(cache, lens, top, qr, o, hot.alloc_cache_attn_workspace(cache, m.Hq, top))
    return x[newest] + o.view(B, -1) @ m.back, whole[newest]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--items", type=int, default=20000)
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args(argv)
    rng = np.random.RandomState(a.seed)
    m = Encoder(a.items, seed=a.seed)
    losses = []

    def batch():
        # histories walk through the items: the next one is mostly the neighbour of the last
        lengths = [int(n) for n in rng.randint(2, 60, a.users)]
        items = np.concatenate([(rng.randint(a.items) + np.cumsum(1 + (rng.rand(n) < 0.1))) % a.items for n in lengths])
        return lengths, torch.from_numpy(items).to(DEV)
    for step in range(a.steps):
        lengths, items = batch()
        others = torch.from_numpy(rng.randint(0, a.items, items.numel())).to(DEV)
        losses.append(train_step(m, lengths, items, others, lr=0.5, row_lr=100.0))
        print("step %d: %d users, %d items, loss %.4f" % (step, a.users, items.numel(), losses[-1]), flush=True)
    one, whole = serve(m, *batch())
    off = float((one - whole).abs().max() / whole.abs().max())
    print("newest items from the cache against whole histories: %.2g off" % off, flush=True)
    return losses, off


if __name__ == "__main__":
    main()
