"""The operators of a paged cache from their definitions, in 64 bits on the
host, with the error that the kernels may make, and the tests' batches."""
import math

import numpy as np
import torch

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
# half a step of a rounding to the storage type, relative to the value
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


class Batch:
    """Sequences in a block pool [L][2][n_blocks][bs][H][d], values of seed."""

    def __init__(self, dtype, heads, kv_heads, d, bs, q, lens, L=1, seed=0, spare=3, shared=0,
                 table_slack=0, fill=None, device="cuda"):
        self.dtype, self.heads, self.kv_heads, self.d, self.bs = dtype, heads, kv_heads, d, bs
        self.q, self.lens, self.L = list(q), list(lens), L
        g = torch.Generator().manual_seed(seed)
        blocks = [-(-max(n, 0) // bs) for n in lens]
        n_sh = shared // bs
        own = [max(b - n_sh, 0) for b in blocks]
        self.n_blocks = n_sh + sum(own) + spare
        ids = torch.randperm(self.n_blocks, generator=g).tolist()
        width = max(max(blocks), 1) + table_slack
        self.table = torch.full((len(q), width), -1, dtype=torch.int32)
        at = n_sh
        for s, b in enumerate(blocks):
            row = (ids[:n_sh] + ids[at:at + own[s]])[:b]
            at += own[s]
            self.table[s, :b] = torch.tensor(row, dtype=torch.int32)
        t = TORCH[dtype]
        self.pool = torch.randn(L, 2, self.n_blocks, bs, kv_heads, d, generator=g).to(t)
        if fill is not None:                    # what lies in no sequence's slots
            keep = torch.zeros(self.n_blocks, bs, dtype=torch.bool)
            for s, n in enumerate(lens):
                for j in range(max(n, 0)):
                    keep[self.table[s, j // bs], j % bs] = True
            self.pool[:, :, ~keep] = fill
        self.N = sum(q)
        new = torch.randn(self.N, heads + 2 * kv_heads, d, generator=g).to(t)
        self.qh, self.kh, self.vh = new[:, :heads], new[:, heads:heads + kv_heads], new[:, heads + kv_heads:]
        self.new = new
        self.off = np.concatenate([[0], np.cumsum(self.q)]).astype(np.int32)
        self.seed = seed

    def cuda(self):
        """(cache, sequences, q, k, v) on the GPU; q, k, v are views of one tensor."""
        from paper_2609_35139_amd.serving import PagedCache
        cache = PagedCache(self.pool.cuda())
        seqs = cache.sequences(self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                               self.off)
        new = self.new.cuda()
        H, K = self.heads, self.kv_heads
        return cache, seqs, new[:, :H], new[:, H:H + K], new[:, H + K:]

    def slots(self):
        """(sequence, slot) of every new token; a length counts as one within the table."""
        most = self.table.shape[1] * self.bs
        return [(s, min(max(n, 0), most) - nq + i)
                for s, (nq, n) in enumerate(zip(self.q, self.lens)) for i in range(nq)]

    def row(self, s, j):
        """(block, row) of slot j, or None."""
        if j < 0 or j // self.bs >= self.table.shape[1]:
            return None
        b = int(self.table[s, j // self.bs])
        return (b, j % self.bs) if 0 <= b < self.n_blocks else None


def append_oracle(b, layer, theta=1e6, scale=1.0, positions=None, rotate=True):
    """(pool, q_out, bound on pool's error, bound on q_out's) in 64 bits."""
    half = b.d // 2
    slots = b.slots()
    pos = torch.tensor([j for _, j in slots] if positions is None else positions, dtype=torch.float64)
    ang = pos[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / half)
    c, s = scale * ang.cos()[:, None], scale * ang.sin()[:, None]

    def rot(x):
        x = x.double()
        if not rotate:
            return x, torch.zeros_like(x)
        u, w = x[..., :half], x[..., half:]
        y = torch.cat([u * c - w * s, w * c + u * s], -1)
        # the cosine and sine are off by their own rounding (2 units in the
        # last place) and by the reduced angle's (2 pi 2^-25), the products
        # and the sum by three roundings; then the stored result's
        size = scale * (u.abs() + w.abs())
        return y, 2.0 ** -20 * torch.cat([size, size], -1) + HALF[b.dtype] * y.abs()

    k, ek = rot(b.kh)
    q, eq = rot(b.qh)
    pool, err = b.pool.double(), torch.zeros(b.pool.shape, dtype=torch.float64)
    for t, (seq, j) in enumerate(slots):
        at = b.row(seq, j)
        if at is not None:
            pool[layer, 0, at[0], at[1]], err[layer, 0, at[0], at[1]] = k[t], ek[t]
            pool[layer, 1, at[0], at[1]] = b.vh[t].double()
    return pool, q, err, eq


def attend_oracle(b, layer, scale=None, softcap=0.0, slopes=None, lo=None, hi=None, pool=None,
                  q=None, tokens=None):
    """(out, lse, bound on out's error, bound on lse's) in 64 bits, from the
    keys that a query sees alone; of the given tokens (None: all)."""
    scale = 1 / math.sqrt(b.d) if scale is None else scale
    pool = (b.pool if pool is None else pool).double()
    q = (b.qh if q is None else q).double()
    G = b.heads // b.kv_heads
    out = torch.zeros(b.N, b.heads, b.d, dtype=torch.float64)
    lse = torch.full((b.N, b.heads), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    half = HALF[b.dtype]
    most = b.table.shape[1] * b.bs
    slots = b.slots()
    for t in range(b.N) if tokens is None else tokens:
        s, p = slots[t]
        n = min(max(b.lens[s], 0), most)
        a = 0 if lo is None else max(int(lo[t]), 0)
        e = min(p + 1 if hi is None else int(hi[t]), n)
        at = [(j, b.row(s, j)) for j in range(a, e)]
        at = [(j, r) for j, r in at if r is not None]
        if not at:
            continue
        j = torch.tensor([x for x, _ in at], dtype=torch.float64)
        blk = torch.tensor([r[0] for _, r in at])
        row = torch.tensor([r[1] for _, r in at])
        K, V = pool[layer, 0, blk, row], pool[layer, 1, blk, row]        # [n][Hkv][d]
        for h in range(b.heads):
            k, v = K[:, h // G], V[:, h // G]
            x = scale * (k @ q[t, h])
            # fp32 sums of d products, then a few roundings of the score
            e_s = scale * (k.abs() @ q[t, h].abs()) * (b.d + 8) * 2.0 ** -24
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                e_s = e_s + softcap * 2.0 ** (-20 if b.dtype == "bf16" else -22)
            if slopes is not None:
                x = x - slopes[h] * (p - j).abs()
                e_s = e_s + 4 * 2.0 ** -24 * (x.abs() + abs(slopes[h]) * (p - j).abs())
            m = x.max()
            w = torch.exp(x - m)
            l = w.sum()
            o = (w / l) @ v
            out[t, h], lse[t, h] = o, m + torch.log(l)
            # a weight is off by its score's error (twice: itself and the sum),
            # the exponential's and the joined parts' roundings, and for bf16
            # by its rounding for the product, which the sum shares; then the
            # result's rounding
            e = float(e_s[torch.isfinite(e_s)].max()) if torch.isfinite(e_s).any() else 0.0
            e += 2.0 ** -21 * (1 + float(x.abs().max()) if torch.isfinite(x).all() else 1.0)
            rel = 2 * e + 2.0 ** -16 + (half if b.dtype == "bf16" else 0.0)
            tol[t, h] = rel * ((w / l) @ v.abs() + o.abs()) + half * o.abs()
            ltol[t, h] = rel
    return out, lse, tol, ltol


def assert_within(got, ref, tol, what):
    got = got.double().cpu()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), what
    over = ((got - ref).abs() - tol)[fine]
    share = ((got - ref).abs() / tol.clamp_min(1e-300))[fine]
    print(f"[{what}] worst share of the bound {float(share.max()) if share.numel() else 0:.3f}", flush=True)
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()))
