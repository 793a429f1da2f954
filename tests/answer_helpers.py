"""The operators that keep an answer going, from their definitions in 64 bits on
the host, with the error that the kernels may make."""
import bisect
import itertools
import math

import numpy as np
import torch


def weigh_oracle(b, layer, lse, weights, scale=None, softcap=0.0, slopes=None, lo=None, hi=None):
    """(weights after the call, bound on their error): serving_helpers.Batch b, lse fp32
    [N][heads], weights fp32 [L][S][Hkv][slots]."""
    scale = 1 / math.sqrt(b.d) if scale is None else scale
    pool, q, lse = b.pool.double(), b.qh.double(), lse.double()
    out = weights.double().clone()
    G = b.heads // b.kv_heads
    tol = torch.zeros_like(out)
    rows = torch.zeros_like(out)
    most = b.table.shape[1] * b.bs
    # (slots count from the length, also where it passes the table)
    at = [(s, max(n, 0) - nq + i) for s, (nq, n) in enumerate(zip(b.q, b.lens)) for i in range(nq)]
    for t, (s, p) in enumerate(at):
        n = min(max(b.lens[s], 0), most)
        a = 0 if lo is None else max(int(lo[t]), 0)
        e = min(p + 1 if hi is None else int(hi[t]), n)
        seen = [(j, b.row(s, j)) for j in range(a, e)]
        seen = [(j, r) for j, r in seen if r is not None]
        if not seen:
            continue
        slot = torch.tensor([j for j, _ in seen])
        K = pool[layer, 0, torch.tensor([r[0] for _, r in seen]), torch.tensor([r[1] for _, r in seen])]
        for h in range(b.heads):
            if lse[t, h] == -math.inf:
                continue
            k = K[:, h // G]
            x = scale * (k @ q[t, h])
            # an fp32 sum of d products, as in the attention's bound
            off = scale * (k.abs() @ q[t, h].abs()) * (b.d + 8) * 2.0 ** -24
            size = x.abs()
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                off = off + softcap * 2.0 ** (-20 if b.dtype == "bf16" else -22)
            if slopes is not None:
                size = size + abs(slopes[h]) * (p - slot).abs()
                x = x - slopes[h] * (p - slot).abs()
            w = torch.exp(x - lse[t, h])
            # the exponent: the scale's rounding, the product's, the distance's and the
            # sums', each at most 2^-24 of the largest number in it (score, distance, lse);
            # the exponential's and the factor's own, 2^-22 in all
            rel = off + 5 * 2.0 ** -24 * (size + x.abs() + lse[t, h].abs()) + 2.0 ** -22
            out[layer, s, h // G, slot] += w
            tol[layer, s, h // G, slot] += w * rel
            rows[layer, s, h // G, slot] += 1
    # sums of non-negative numbers: each addition is off by half a step of a partial sum
    return out, tol + (rows + 8) * 2.0 ** -24 * out.abs()


def choose_oracle(weights, lens, slots, budget, first=0, recent=0, budgets=None):
    """(kept, kept_lens) by sorting, of weights [L][S][H][slots]."""
    L, S, H, _ = weights.shape
    kept = np.full((L, S, H, budget), -1, dtype=np.int32)
    kept_lens = np.zeros(S, dtype=np.int32)
    for s in range(S):
        n = min(max(int(lens[s]), 0), slots)
        m = min(n, budget if budgets is None else min(max(int(budgets[s]), 0), budget))
        r = min(recent, m)
        f = min(first, m - r)
        kept_lens[s] = m
        for l in range(L):
            for h in range(H):
                w = weights[l, s, h, :n].double().numpy()
                w = np.where(np.isnan(w), -np.inf, w)
                middle = sorted(range(f, n - r), key=lambda j: (-w[j], j))[:m - f - r]
                kept[l, s, h, :m] = sorted(list(range(f)) + middle + list(range(n - r, n)))
    return kept, kept_lens


def compact_oracle(pool, table, lens, kept, kept_lens, weights=None, table_out=None):
    """(pool, weights) after the move: pool [L][2][blocks][bs][H][d], host tensors."""
    pool, src = pool.clone(), pool
    L, _, n_blocks, bs, H, _ = pool.shape
    w = None if weights is None else weights.clone()
    to = table if table_out is None else table_out
    slots = table.shape[1] * bs
    for s in range(table.shape[0]):
        n = min(max(int(lens[s]), 0), slots)
        m = min(max(int(kept_lens[s]), 0), kept.shape[3])
        for l in range(L):
            for h in range(H):
                if w is not None:
                    w[l, s, h, m:n] = 0
                for i in range(m):
                    j = int(kept[l, s, h, i])
                    if not 0 <= j < n:
                        continue
                    if w is not None:
                        w[l, s, h, i] = weights[l, s, h, j]
                    if i >= to.shape[1] * bs:
                        continue
                    a, c = int(table[s, j // bs]), int(to[s, i // bs])
                    if 0 <= a < n_blocks and 0 <= c < n_blocks:
                        pool[l, :, c, i % bs, h] = src[l, :, a, j % bs, h]
    return pool, w


def sample_oracle(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens, log-probabilities) of host logits [R][V]; settings are numbers or [R]."""
    R, V = logits.shape

    def per_row(x, dtype):
        x = x.numpy() if isinstance(x, torch.Tensor) else x
        return np.broadcast_to(np.asarray(x, dtype=dtype).astype(np.float64), (R,))

    T, P, M = (per_row(x, np.float32) for x in (temperature, top_p, min_p))
    K = per_row(top_k, np.int32)
    tokens, log_p = np.zeros(R, dtype=np.int32), np.zeros(R)
    for r in range(R):
        x = logits[r].double().numpy()
        x = np.where(np.isnan(x), -np.inf, x)
        order = np.argsort(-x, kind="stable")
        n = int(np.count_nonzero(x > -np.inf))
        if n == 0:
            tokens[r], log_p[r] = -1, -np.inf
            continue
        if not T[r] > 0 or not P[r] > 0 or not M[r] <= 1:
            tokens[r] = order[0]
            continue
        if K[r] > 0:
            n = min(n, int(K[r]))
        here = x[order[:n]]
        if here[0] == np.inf:
            p = (here == np.inf).astype(np.float64)
        else:
            p = np.exp((here - here[0]) / T[r])
        mass = np.cumsum(p)
        stays = p >= M[r]
        if P[r] < 1:
            stays &= np.concatenate([[0.0], mass[:-1]]) < P[r] * mass[-1]
        stays[0] = True
        index, p = order[:n][stays], p[stays]
        by_index = np.argsort(index, kind="stable")
        index, p = index[by_index], p[by_index]
        number = float(u[r])
        number = number if number > 0 else 0.0
        if len(p) <= 20000:
            # whole numbers of 2^-80 and of 2^-149 (any fp32 number): equal logits put u times
            # the sum exactly on a border, where a rounded sum would fall on either side
            mass = list(itertools.accumulate(int(v) for v in np.ldexp(p, 80)))
            share = int(math.ldexp(min(number, 2.0), 149)) * mass[-1]
            i = bisect.bisect_right([m << 149 for m in mass], share)
        else:
            mass = np.cumsum(p)
            i = int(np.count_nonzero(mass <= number * mass[-1]))
        i = min(i, int(np.flatnonzero(p > 0)[-1]))
        mass = np.cumsum(p)
        tokens[r] = index[i]
        log_p[r] = math.log(p[i]) - math.log(mass[-1])
    return tokens, log_p


# log_probs: the weights are off by half a step of 2^-44 (2^-42 for more than 2^18 logits)
# and 2^-44 of themselves, their sum is at least 1; then one rounding to fp32.
def log_prob_bound(ref, vocab):
    step = 2.0 ** -45 if vocab <= 1 << 18 else 2.0 ** -43
    return vocab * step + 2.0 ** -43 + 2.0 ** -24 * np.abs(ref)
