"""The operators that keep an answer going, and what they must compute.

A request's repaired cache grows with every token of the answer, and the target
model's logits have to become that token.  Four operators:

``weigh``    how much attention every cached slot receives: the probabilities
             of a call's queries, summed over the queries and the query heads
             of a KV head, are added to the slot's weight (one layer);
``choose``   which slots stay when a sequence is over its budget, for every
             layer and KV head by itself: the first ones, the recent ones, and
             of the others those of the largest weight (ties: the lowest slot);
``compact``  their keys, values and weights moved to the front, in place or
             into other blocks (all layers);
``sample``   a token from the logits of every row by temperature, top-k, top-p
             and min-p and a given random number, with its log-probability.

A case names an operator and its sizes; lengths follow from ``shape``, values
from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
# query heads, KV heads, head_dim of the repository's targets, and of a small fp32 one
HEADS = {"qwen3b": (16, 2, 128), "llama8b": (32, 8, 128), "tiny": (4, 2, 64)}


def _heads(target):
    return HEADS[target] if isinstance(target, str) else target


def _weigh(name, target, seqs, q, length, shape, dtype="bf16", page=16, mask="causal", cap=0.0,
           bias=False):
    heads, kv_heads, head_dim = _heads(target)
    return {"name": name, "op": "weigh", "dtype": dtype, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "seqs": seqs, "q_lo": q[0], "q_hi": q[1],
            "len_lo": length[0], "len_hi": length[1], "shape": shape, "mask": mask, "cap": cap,
            "bias": bias}


def _keep(name, op, target, layers, seqs, length, budget, first, recent, shape, dtype="bf16",
          page=16, moved=False):
    heads, kv_heads, head_dim = _heads(target)
    return {"name": name, "op": op, "dtype": dtype, "layers": layers, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "seqs": seqs, "len_lo": length[0],
            "len_hi": length[1], "budget": budget, "first": first, "recent": recent,
            "shape": shape, "moved": moved}


def _sample(name, rows, vocab, dtype, temperature, top_k, top_p, min_p, mixed=False, spread=2.0):
    return {"name": name, "op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab,
            "temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "mixed": mixed, "spread": spread}


def listed():
    return [
        # one token over eight repaired passages: latency
        _weigh("weigh-1x4096", "qwen3b", 1, (1, 1), (4095, 4095), 1),
        # a decoding step of a batch whose lengths differ widely: reading the keys
        _weigh("weigh-64-ragged-8b", "llama8b", 64, (1, 1), (64, 16000), 2),
        # the questions' tokens weigh the passages before the answer begins
        _weigh("weigh-questions-8b", "llama8b", 5, (17, 333), (1177, 8001), 3),
        # a whole uncached prompt weighs what came before it and itself: computing
        _weigh("weigh-prompt-8b", "llama8b", 1, (8192, 8192), (4096, 4096), 4, page=64),
        # fp32, capped scores with a bias by distance, intervals of documents, odd lengths
        _weigh("weigh-f32-documents", "tiny", 7, (1, 77), (30, 1201), 5, dtype="f32", page=8,
               mask="documents", cap=30.0, bias=True),
        # one request over its budget, all layers
        _keep("choose-1x4096", "choose", "qwen3b", 36, 1, (4096, 4096), 2048, 4, 256, 6),
        # a ragged batch, some sequences within their budget
        _keep("choose-8-ragged-8b", "choose", "llama8b", 32, 8, (900, 30011), 4001, 4, 512, 7),
        # the same request's pages compacted in place
        _keep("compact-1x4096", "compact", "qwen3b", 36, 1, (4096, 4096), 2048, 4, 256, 6),
        # a ragged batch into fresh blocks, where its passages were shared with others
        _keep("compact-5-moved-8b", "compact", "llama8b", 16, 5, (300, 3001), 1023, 1, 100, 8,
              moved=True),
        # the next token of one request: latency
        _sample("sample-1-top-k", 1, 151936, "bf16", 0.7, 20, 0.8, 0.0),
        # a batch of requests with settings of their own, fp32 logits
        _sample("sample-256-mixed", 256, 151936, "f32", 1.0, 0, 1.0, 0.0, mixed=True),
        # 33 samples by top-p and min-p alone, of flat logits
        _sample("sample-33-top-p", 33, 128256, "bf16", 1.3, 0, 0.95, 0.001, spread=1.0),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    """A case of the listed ranges: one to 64 sequences, one to 8,192 queries over one to 131,072
    slots; one to 36 layers of up to 32,768 slots; one to 256 rows of 1,000 to 152,000 logits."""
    op = rng.choice(["weigh", "weigh", "weigh", "choose", "choose", "compact", "compact",
                     "sample", "sample", "sample"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    size = 4 if dtype == "f32" else 2
    if op == "sample":
        rows, vocab = _log(rng, 1, 256), _log(rng, 1000, 152000)
        return dict(_sample("drawn", rows, vocab, dtype, round(rng.uniform(0.3, 1.5), 2),
                            rng.choice([0, 0, 1, 5, 20, 50, 200, vocab // 3]),
                            rng.choice([1.0, 1.0, 0.5, 0.8, 0.95, 0.99]),
                            rng.choice([0.0, 0.0, 0.0, 0.05, 0.001]), mixed=rng.random() < 0.4,
                            spread=round(rng.uniform(0.5, 3.0), 2)))
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    head_dim = rng.choice([64, 128, 128, 128, 96, 256])
    page = rng.choice([1, 8, 16, 16, 16, 64, 256])
    seqs = _log(rng, 1, 64)
    shape = rng.randrange(1 << 30)
    if op == "weigh":
        heads = kv_heads * rng.choice([1, 2, 4, 5, 7, 8])
        q_hi = 1 if rng.random() < 0.5 else _log(rng, 2, min(8192, 12000 // seqs))
        pairs = int(5e11) // (2 * head_dim * heads) // (8 if dtype == "f32" else 1)
        while seqs * q_hi * q_hi > pairs // 2:
            q_hi //= 2
        budget = (400 << 20) // (kv_heads * head_dim * size) // seqs
        most = max(1, min(131072, budget, pairs // 2 // (seqs * q_hi)))
        len_hi = _log(rng, min(16, most), most)
        return dict(_weigh("drawn", (heads, kv_heads, head_dim), seqs, (rng.randint(1, q_hi), q_hi),
                           (rng.randint(0, len_hi), len_hi), shape, dtype=dtype, page=page,
                           mask=rng.choice(["causal", "causal", "documents", "prefix"]),
                           cap=rng.choice([0.0, 0.0, 15.0, 50.0]), bias=rng.random() < 0.3))
    layers = _log(rng, 1, 36)
    budget = (350 << 20) // (2 * kv_heads * head_dim * size) // (layers * seqs)
    if op == "choose":
        budget = (14 << 20) // (layers * seqs * kv_heads)
    most = max(16, min(32768, budget))
    len_hi = _log(rng, 16, most)
    keep = rng.randint(1, len_hi)
    first = min(keep, rng.choice([0, 1, 4, 100]))
    return dict(_keep("drawn", op, (kv_heads, kv_heads, head_dim), layers, seqs,
                      (rng.randint(1, len_hi), len_hi), keep, first,
                      rng.randint(0, keep - first), shape, dtype=dtype, page=page,
                      moved=op == "compact" and rng.random() < 0.4))


def _lengths(case):
    """(new tokens, length) of every sequence."""
    rng = random.Random(case["shape"])
    q = [rng.randint(case["q_lo"], case["q_hi"]) if "q_lo" in case else 0
         for _ in range(case["seqs"])]
    return q, [n + _log(rng, case["len_lo"] + 1, case["len_hi"] + 1) - 1 for n in q]


def _intervals(case, q, total):
    """Slots [lo, hi) that every query sees, in order of the queries."""
    rng = random.Random(case["shape"] + 1)
    lo, hi = [], []
    for nq, n in zip(q, total):
        edges = sorted(rng.randrange(n) for _ in range(6))
        for i in range(nq):
            p = n - nq + i
            if case["mask"] == "documents":       # from the start of a document; some see nothing
                a = rng.choice([e for e in edges if e <= p] or [0])
                lo.append(a)
                hi.append(a if rng.random() < 1 / 16 else p + 1)
            else:                                 # causal, but all of the first two thirds
                lo.append(0)
                hi.append(max(p + 1, 2 * n // 3))
    return lo, hi


def _table(lens, page, host, first_id=0):
    """(rows of block ids, blocks) of sequences of these lengths, in a random order."""
    need = [-(-n // page) for n in lens]
    ids = list(range(first_id, first_id + sum(need)))
    host.shuffle(ids)
    rows, at = [], 0
    for n in need:
        rows.append(ids[at:at + n] + [-1] * (max(need) - n))
        at += n
    return rows, sum(need)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, g)
    q, total = _lengths(case)
    dt, ps, Hkv, d = TORCH[case["dtype"]], case["page"], case["kv_heads"], case["head_dim"]
    S, L = case["seqs"], case.get("layers", 1)
    rows, used = _table(total, ps, host)
    st = {"case": dict(case), "q": q, "total": total, "rows": rows, "table": _int32(rows),
          "lens": _int32(total)}
    width = st["table"].shape[1] * ps
    if case["op"] == "weigh":
        return _prepare_weigh(case, st, g, used)
    # what a few thousand queries left: a few slots hold most of the weight, some none, and some
    # (repeated tokens) the same
    w = torch.empty(L, S, Hkv, width, device="cuda").normal_(0.0, 2.0, generator=g).exp_()
    w *= torch.empty_like(w).uniform_(generator=g) > 0.1
    same = torch.empty_like(w).uniform_(generator=g) < 0.05
    st["weights"] = torch.where(same, torch.full_like(w, 0.125), w)
    st["kept_lens"] = torch.clamp(st["lens"], max=case["budget"])
    if case["op"] == "choose":
        st["kept"] = torch.empty(L, S, Hkv, case["budget"], dtype=torch.int32, device="cuda")
        n_blocks = used
    else:
        st["kept"], _ = _plain_choose(st)
        n_blocks, st["table_out"] = used + 3, None
        if case["moved"]:
            out, more = _table([min(n, case["budget"]) for n in total], ps, host, used)
            n_blocks, st["table_out"] = used + more + 3, _int32(out)
    # (no key is read by the choice: its cache is a layout and nothing else)
    blocks = n_blocks if case["op"] == "compact" else 1
    pool = torch.empty(L, 2, blocks, ps, Hkv, d, dtype=dt, device="cuda")
    st["pool"] = pool.normal_(generator=g) if case["op"] == "compact" else pool
    if own:
        from paper_2609_35139_amd.serving import PagedCache
        st["cache"] = PagedCache(st["pool"])
        st["seqs"] = st["cache"].sequences(st["table"], st["lens"])
    return st


def _prepare_weigh(case, st, g, used):
    q, total = st["q"], st["total"]
    dt, ps, H, Hkv, d = (TORCH[case["dtype"]], case["page"], case["heads"], case["kv_heads"],
                         case["head_dim"])
    pool = torch.empty(1, 2, used + 3, ps, Hkv, d, dtype=dt, device="cuda").normal_(generator=g)
    spread = torch.empty(Hkv, d, device="cuda").uniform_(math.log(0.5), math.log(8.0), generator=g)
    pool[:, 0] *= spread.exp().to(dt)
    N = sum(q)
    off = [0]
    for n in q:
        off.append(off[-1] + n)
    st.update(pool=pool, off=off, lo=None, hi=None, slopes=None,
              qh=torch.empty(N, H, d, dtype=dt, device="cuda").normal_(generator=g),
              weights=torch.empty(1, case["seqs"], Hkv, st["table"].shape[1] * ps,
                                  device="cuda").uniform_(generator=g))
    if case["mask"] != "causal":
        lo, hi = _intervals(case, q, total)
        st["lo"], st["hi"] = _int32(lo), _int32(hi)
    if case["bias"]:
        st["slopes"] = [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]
    # what the attention of these queries left: the logarithm of each row's sum
    lse = torch.empty(N, H, device="cuda")
    for s, a, b, x in _scores(st):
        G = x.shape[0] // (b - a)
        lse[off[s]:off[s + 1], a * G:b * G] = torch.logsumexp(x, 2).t()
    st["lse"] = lse
    if own:
        from paper_2609_35139_amd.serving import PagedCache
        st["cache"] = PagedCache(pool)
        st["seqs"] = st["cache"].sequences(st["table"], st["lens"], off)
    return st


def _prepare_sample(case, g):
    R, V = case["rows"], case["vocab"]
    # most logits lie in one wide heap, a few tokens (others in every row) stand out of it
    x = torch.empty(R, V, device="cuda").normal_(0.0, case["spread"], generator=g)
    n = min(V, 64)
    at = torch.empty(R, n, device="cuda").uniform_(0, V, generator=g).long().clamp_max(V - 1)
    lift = torch.empty(R, n, device="cuda").exponential_(generator=g) * 2 + 3 * case["spread"]
    x.scatter_add_(1, at, lift)
    st = {"case": dict(case), "logits": x.to(TORCH[case["dtype"]]),
          "u": torch.empty(R, device="cuda").uniform_(generator=g)}
    for name in ("temperature", "top_k", "top_p", "min_p"):
        st[name] = case[name]
    if case["mixed"]:
        pick = torch.randint(0, 6, (R,), generator=g, device="cuda")
        st["temperature"] = torch.tensor([0.0, 0.3, 0.7, 1.0, 1.0, 1.5], device="cuda")[pick]
        st["top_k"] = _int32([0, 1, 20, 50, 0, 1500])[(pick * 5 + 1) % 6]
        st["top_p"] = torch.tensor([1.0, 0.9, 0.95, 1.0, 0.8, 1.0], device="cuda")[(pick + 2) % 6]
        st["min_p"] = torch.tensor([0.0, 0.0, 0.05, 0.0, 0.0, 0.01], device="cuda")[pick]
    return st


def run(st):
    op = st["case"]["op"]
    if own:
        c = st["case"]
        if op == "weigh":
            st["cache"].weigh(0, st["seqs"], st["qh"], st["lse"], st["weights"], softcap=c["cap"],
                              slopes=st["slopes"], lo=st["lo"], hi=st["hi"])
            return [st["weights"]]
        if op == "choose":
            return list(st["cache"].choose(st["seqs"], st["weights"], c["budget"], first=c["first"],
                                           recent=c["recent"], kept=st["kept"]))
        if op == "compact":
            st["cache"].compact(st["seqs"], st["kept"], st["kept_lens"], weights=st["weights"],
                                block_table=st["table_out"])
            return [st["pool"], st["weights"]]
        from paper_2609_35139_amd.serving import sample
        return list(sample(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"],
                           top_p=st["top_p"], min_p=st["min_p"]))
    if op == "weigh":
        return _plain_weigh(st)
    if op == "choose":
        return list(_plain_choose(st))
    return _plain_compact(st) if op == "compact" else _plain_sample(st)


def _scores(st):
    """For every sequence s and range [a, b) of KV heads: (s, a, b, scores [(b - a) G, queries,
    keys]) in 32 bits, -inf where a query does not see the key."""
    c = st["case"]
    H, Hkv, d, ps = c["heads"], c["kv_heads"], c["head_dim"], c["page"]
    G = H // Hkv
    for s, (nq, n) in enumerate(zip(st["q"], st["total"])):
        o = st["off"][s]
        key = st["pool"][0, 0, st["table"][s, :-(-n // ps)].long()].reshape(-1, Hkv, d)[:n]
        j = torch.arange(n, device="cuda")
        p = torch.arange(n - nq, n, device="cuda")
        if st["lo"] is None:
            see = j[None] <= p[:, None]
        else:
            see = (j[None] >= st["lo"][o:o + nq, None]) & (j[None] < st["hi"][o:o + nq, None])
        step = max(1, (1 << 29) // (G * nq * n))
        for a in range(0, Hkv, step):
            b = min(Hkv, a + step)
            x = st["qh"][o:o + nq, a * G:b * G].float().transpose(0, 1).reshape(b - a, G * nq, d)
            x = x @ key[:, a:b].float().permute(1, 2, 0).contiguous()
            x = (x * (1.0 / math.sqrt(d))).view((b - a) * G, nq, n)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if st["slopes"] is not None:
                slope = torch.tensor(st["slopes"][a * G:b * G], device="cuda")
                x = x - slope[:, None, None] * (p[:, None] - j[None]).abs()
            yield s, a, b, x.masked_fill(~see, -math.inf)


def _plain_weigh(st):
    for s, a, b, x in _scores(st):
        nq, n = st["q"][s], st["total"][s]
        G = x.shape[0] // (b - a)
        lse = st["lse"][st["off"][s]:st["off"][s + 1], a * G:b * G].t()[..., None]
        w = (x - torch.where(lse > -math.inf, lse, torch.zeros_like(lse))).exp()
        st["weights"][0, s, a:b, :n] += w.view(b - a, G * nq, n).sum(1)
    return [st["weights"]]


def _plain_choose(st):
    c, w = st["case"], st["weights"]
    width = w.shape[3]
    n = st["lens"].long()[None, :, None, None]
    most = torch.clamp(n, max=c["budget"])
    j = torch.arange(width, device="cuda")
    recent = torch.clamp(most, max=c["recent"])
    first = torch.minimum(most - recent, torch.full_like(most, c["first"]))
    w = w.masked_fill((j < first) | (j >= n - recent), math.inf).masked_fill(j >= n, -1.0)
    order = w.sort(dim=3, descending=True, stable=True).indices[..., :c["budget"]]
    if order.shape[3] < c["budget"]:
        order = torch.nn.functional.pad(order, (0, c["budget"] - order.shape[3]))
    i = torch.arange(c["budget"], device="cuda")
    kept = order.masked_fill(i >= most, width).sort(dim=3).values
    return kept.masked_fill(i >= most, -1).int(), st["kept_lens"].clone()


def _plain_compact(st):
    c, w, pool = st["case"], st["weights"], st["pool"]
    L, S, H, B = st["kept"].shape
    kept, ps = st["kept"].long(), c["page"]
    i = torch.arange(B, device="cuda")
    valid = (i < st["kept_lens"].long()[None, :, None, None]).expand(L, S, H, B)
    layer, seq, head, to = valid.nonzero(as_tuple=True)
    at = kept[valid]
    out = st["table"] if st["table_out"] is None else st["table_out"]
    src = pool[layer, :, st["table"].long()[seq, at // ps], at % ps, head]
    pool[layer, :, out.long()[seq, to // ps], to % ps, head] = src
    held = w[layer, seq, head, at]
    j = torch.arange(w.shape[3], device="cuda")
    w.masked_fill_(j < st["lens"].long()[None, :, None, None], 0.0)
    w[layer, seq, head, to] = held
    return [pool, w]


def _column(x, rows):
    """A setting of every row: [rows][1] in 64 bits."""
    if not isinstance(x, torch.Tensor):
        x = torch.full((rows,), x, device="cuda", dtype=torch.float32)   # as the call takes it
    return x.double()[:, None]


def _plain_sample(st):
    x = st["logits"].double()
    R, V = x.shape
    T, k = _column(st["temperature"], R), _column(st["top_k"], R)
    top_p, min_p = _column(st["top_p"], R), _column(st["min_p"], R)
    greedy = T <= 0
    x, order = x.sort(dim=1, descending=True, stable=True)
    rank = torch.arange(V, device="cuda")[None]
    p = ((x - x[:, :1]) / torch.where(greedy, torch.ones_like(T), T)).exp()
    limit = torch.where(greedy, torch.ones_like(k), torch.where(k <= 0, torch.full_like(k, V), k))
    p = p.masked_fill(rank >= limit, 0.0)
    before = torch.nn.functional.pad(p.cumsum(1), (1, 0))
    stays = (before[:, :V] < top_p * before[:, V:]) | (top_p >= 1)
    stays = (stays & (p >= min_p)) | (rank == 0)
    p = torch.zeros_like(p).scatter_(1, order, p.masked_fill(~stays, 0.0))
    upto = p.cumsum(1)
    total = upto[:, -1:]
    token = torch.searchsorted(upto, st["u"].double()[:, None] * total, right=True)
    token = torch.minimum(token, torch.searchsorted(upto, total))   # the last one that stays
    log_p = (p.gather(1, token) / total).log()
    return [token[:, 0].int(), log_p[:, 0].float()]


def work(case):
    """Weigh: every key that some query sees, every query and its sum once in, every weight of a
    sequence in and out, 2 d operations for each pair of query head and key.  Choose: the weights
    of the sequences over their budget in, the list out, a comparison for each weight.  Compact:
    what moves in and out, the list and the weights in, the weights out.  Sample: every logit
    once, an exponential's worth of four operations for each."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + 12 * case["rows"], "flops": 4 * n}
    q, total = _lengths(case)
    Hkv, d = case["kv_heads"], case["head_dim"]
    if case["op"] == "weigh":
        H, N = case["heads"], sum(q)
        if case["mask"] == "causal":
            pairs = sum(nq * (n - nq) + nq * (nq + 1) // 2 for nq, n in zip(q, total))
            keys = sum(total)
        else:
            lo, hi = _intervals(case, q, total)
            pairs = sum(b - a for a, b in zip(lo, hi))
            keys, i = 0, 0
            for nq in q:
                seen = [(a, b) for a, b in zip(lo[i:i + nq], hi[i:i + nq]) if b > a]
                keys += max(b for _, b in seen) - min(a for a, _ in seen) if seen else 0
                i += nq
        return {"bytes": size * d * (N * H + keys * Hkv) + 4 * N * H + 8 * keys * Hkv,
                "flops": 2 * d * H * pairs}
    rows, B = case["layers"] * Hkv, case["budget"]
    kept = sum(min(n, B) for n in total)
    if case["op"] == "choose":
        over = sum(n for n in total if n > B)
        return {"bytes": 4 * rows * (over + case["seqs"] * B), "flops": rows * over}
    moved = kept if case["moved"] else sum(B - case["first"] for n in total if n > B)
    return {"bytes": rows * (4 * d * size * moved + 4 * kept + 4 * kept + 4 * sum(total)),
            "flops": rows * kept}


def exact(case, seed):
    if case["op"] == "choose":
        return None                    # whole numbers alone
    st = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_sample(st)
    if case["op"] == "compact":
        return _exact_compact(st)
    if work(case)["flops"] > 2e12:
        return None
    H, Hkv, d, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    out = st["weights"].double()
    slopes = torch.tensor(st["slopes"] or [0.0] * H, dtype=torch.float64, device="cuda")
    for s in range(case["seqs"]):
        n, nq = st["total"][s], st["q"][s]
        where = torch.tensor([st["rows"][s][b] for b in range(-(-n // ps))], device="cuda")
        key = st["pool"][0, 0, where].flatten(0, 1)[:n].double().permute(1, 2, 0).contiguous()
        step = max(1, (1 << 28) // (n * H))
        for a in range(0, nq, step):
            b = min(nq, a + step)
            rows = slice(st["off"][s] + a, st["off"][s] + b)
            x = st["qh"][rows].double().view(b - a, Hkv, -1, d).permute(1, 2, 0, 3)
            z = (x.reshape(Hkv, -1, d) @ key).view(H, b - a, n) / d ** 0.5
            if case["cap"]:
                z = torch.tanh(z / case["cap"]) * case["cap"]
            here = torch.arange(n - nq + a, n - nq + b, device="cuda").double()[:, None]
            at = torch.arange(n, device="cuda").double()[None]
            z = z - slopes[:, None, None] * (here - at).abs()
            if st["hi"] is None:
                hidden = at > here
            else:
                hidden = (at < st["lo"][rows, None]) | (at >= st["hi"][rows, None])
            share = torch.exp(z - st["lse"][rows].double().t()[..., None])
            share[:, hidden] = 0
            out[0, s, :, :n] += share.view(Hkv, -1, n).sum(1)
    return [out]


def _exact_compact(st):
    """Row by row in slot numbers of the whole pool."""
    c, pool, w = st["case"], st["pool"].clone(), st["weights"].clone()
    ps = c["page"]
    table = st["table"].tolist()
    out = table if st["table_out"] is None else st["table_out"].tolist()
    for s in range(c["seqs"]):
        n, m = st["total"][s], int(st["kept_lens"][s])
        src = torch.tensor([table[s][j // ps] * ps + j % ps for j in range(n)], device="cuda")
        dst = torch.tensor([out[s][j // ps] * ps + j % ps for j in range(m)], device="cuda")
        for h in range(c["kv_heads"]):
            for layer in range(c["layers"]):
                at = st["kept"][layer, s, h, :m].long()
                old = st["pool"][layer, :, :, :, h].reshape(2, -1, c["head_dim"])[:, src[at]]
                pool[layer, :, dst // ps, dst % ps, h] = old
                w[layer, s, h, :n] = 0
                w[layer, s, h, :m] = st["weights"][layer, s, h, at]
    return [pool.double(), w.double()]


def _exact_sample(st):
    """Row by row on the host, from the order of the logits."""
    R, V = st["logits"].shape
    logits, u = st["logits"].double().cpu().numpy(), st["u"].double().cpu().numpy()
    T, k, top_p, min_p = (_column(st[x], R)[:, 0].cpu().numpy()
                          for x in ("temperature", "top_k", "top_p", "min_p"))
    tokens, log_p = [], []
    for r in range(R):
        order = np.argsort(-logits[r], kind="stable")
        n = 1 if T[r] <= 0 else V if k[r] <= 0 else min(V, int(k[r]))
        p = np.exp((logits[r][order[:n]] - logits[r][order[0]]) / (T[r] if T[r] > 0 else 1.0))
        if top_p[r] < 1:
            mass = np.cumsum(p)
            n = 1 + int(np.count_nonzero(mass[:-1] < top_p[r] * mass[-1]))
        n = max(1, min(n, int(np.count_nonzero(p >= min_p[r]))))
        here = np.sort(order[:n])
        p = np.exp((logits[r][here] - logits[r][order[0]]) / (T[r] if T[r] > 0 else 1.0))
        mass = np.cumsum(p)
        i = min(n - 1, int(np.count_nonzero(mass <= u[r] * mass[-1])))
        tokens.append(int(here[i]))
        log_p.append(math.log(p[i]) - math.log(mass[-1]))
    return [torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            torch.tensor(log_p, dtype=torch.float64, device="cuda")]
