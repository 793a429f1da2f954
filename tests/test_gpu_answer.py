"""cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample on the GPU against
their definitions in 64 bits (tests/answer_helpers.py): weights within bounds
derived there from the roundings, everything else exactly."""
import math

import numpy as np
import pytest
import torch

from answer_helpers import (choose_oracle, compact_oracle, log_prob_bound, sample_oracle,
                            weigh_oracle)
from serving_helpers import TORCH, Batch, assert_within, attend_oracle

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35139_amd import binding
    binding.load()


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


# -------------------------------------------------------------------- weigh
WEIGH = {
    # single tokens: one row of a group, lengths from none to several tiles
    "tokens": dict(dtype="bf16", heads=16, kv_heads=2, d=128, bs=16, q=[1] * 6, lens=[1, 0, 17, 250, 33, 129]),
    "tokens-f32": dict(dtype="f32", heads=4, kv_heads=4, d=96, bs=1, q=[1, 0, 1], lens=[3, 5, 90]),
    # up to 512 rows for a KV head, over few tiles
    "rows": dict(dtype="bf16", heads=6, kv_heads=3, d=64, bs=8, q=[0, 5, 1, 40], lens=[9, 5, 130, 141]),
    "rows-f32": dict(dtype="f32", heads=5, kv_heads=1, d=32, bs=4, q=[7, 30], lens=[7, 150]),
    # prompts of fewer rows than go through LDS, groups that do not divide a step's rows
    "prompt": dict(dtype="bf16", heads=8, kv_heads=2, d=128, bs=16, q=[90, 0, 3], lens=[200, 4, 100]),
    "prompt-odd": dict(dtype="bf16", heads=7, kv_heads=1, d=64, bs=8, q=[61], lens=[170]),
    "prompt-f32": dict(dtype="f32", heads=5, kv_heads=1, d=128, bs=2, q=[60, 2], lens=[60, 300]),
    "short": dict(dtype="bf16", heads=2, kv_heads=2, d=64, bs=4, q=[5, 2, 1], lens=[3, -2, 0]),
}


def _weigh_case(b, layer, seed=0, capture=None, **o):
    """The kernel's weights against the oracle's, both from the oracle's lse in fp32."""
    g = torch.Generator().manual_seed(seed)
    S, width = b.table.shape[0], b.table.shape[1] * b.bs
    prior = torch.rand(b.L, S, b.kv_heads, width, generator=g)
    _, lse, _, _ = attend_oracle(b, layer, **o)
    lse = lse.float()
    ref, tol = weigh_oracle(b, layer, lse, prior, **o)
    cache, seqs, q, _, _ = b.cuda()
    w = prior.cuda()
    k = {n: (_i32(x) if n in ("lo", "hi") else x) for n, x in o.items() if x is not None}
    assert cache.weigh(layer, seqs, q, lse.cuda(), w, **k) is w
    assert_within(w, ref, tol, "weights")
    return w, cache, seqs, q, lse.cuda(), prior, k


@pytest.mark.parametrize("name", WEIGH)
def test_weigh_causal(name):
    b = Batch(L=2, seed=len(name), fill=7.5, **WEIGH[name])
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 1)
    again = prior.cuda()                                 # sums in an order of their own
    cache.weigh(1, seqs, q, lse, again)
    assert torch.equal(again, w)


@pytest.mark.parametrize("name", ["tokens", "rows", "rows-f32", "prompt", "prompt-odd", "prompt-f32"])
@pytest.mark.parametrize("kind", ["intervals", "cap", "slopes", "all"])
def test_weigh_options(name, kind):
    b = Batch(L=1, seed=3 + len(name), **WEIGH[name])
    rng = np.random.default_rng(5)
    o = {}
    if kind in ("intervals", "all"):                     # some rows see nothing, some all, some the end
        lo = rng.integers(-5, 120, b.N)
        o.update(lo=lo.tolist(), hi=(lo + rng.integers(-3, 150, b.N)).tolist())
    if kind in ("cap", "all"):
        o["softcap"] = 2.5
    if kind in ("slopes", "all"):
        o.update(slopes=[0.3 * 2.0 ** -h for h in range(b.heads)], scale=0.2)
    _weigh_case(b, 0, **o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", range(32, 257, 32))
@pytest.mark.parametrize("q", [1, 9, 70])
def test_weigh_every_head_dim(dtype, d, q):
    b = Batch(dtype, 8, 2, d, 16, [q], [q + 75], seed=d + q)
    _weigh_case(b, 0)


@pytest.mark.parametrize("name", ["tokens", "rows", "prompt"])
def test_weigh_does_not_look_at_hidden_keys(name):
    """Infinities and NaN in keys that no query sees, and in blocks that are none, change
    nothing; seen ones change their own slot alone."""
    b = Batch(L=1, seed=9, fill=NAN, **WEIGH[name])
    hi = []
    for (s, p) in b.slots():
        hi.append(min(p + 1, 40))
    for s, n in enumerate(b.lens):
        for j in range(40, max(n, 0)):
            blk, r = b.row(s, j)
            b.pool[0, 0, blk, r] = [INF, -INF, NAN][j % 3]
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 0, hi=hi)
    s = int(np.argmax(b.lens))
    blk, r = b.row(s, 3)
    cache.pool[0, 0, blk, r] = NAN
    w2 = prior.cuda()
    cache.weigh(0, seqs, q, lse, w2, **k)
    touched = torch.isnan(w2)
    assert touched[0, s, :, 3].any() and int(touched.sum()) <= b.kv_heads
    w2[touched] = w[touched]
    assert torch.equal(w2, w)


def test_weigh_blocks_that_are_none_and_lengths_past_the_table():
    b = Batch("bf16", 4, 2, 64, 8, [1, 20], [60, 64], seed=2)
    b.table[0, 3] = -1
    b.table[1, 2] = 1 << 30
    b.lens[1] = 100                                      # eight blocks of the table hold 64
    _weigh_case(b, 0)
    b = Batch("bf16", 8, 1, 64, 8, [70], [90], seed=2)
    b.table[0, 4] = b.n_blocks
    _weigh_case(b, 0)


@pytest.mark.parametrize("q", [1, 30, 80])
def test_weigh_rows_without_a_sum(q):
    """A row whose lse is -inf gives nothing; NaN and +inf stay with what the row sees."""
    b = Batch("bf16", 4, 2, 64, 16, [q, q], [q + 30, q + 50], seed=q)
    _, lse, _, _ = attend_oracle(b, 0)
    cache, seqs, qh, _, _ = b.cuda()
    dead = lse.float().cuda()
    dead[:q] = -INF
    w = cache.new_weights(seqs)
    cache.weigh(0, seqs, qh, dead, w)
    assert torch.equal(w[0, 0], torch.zeros_like(w[0, 0])) and float(w[0, 1].sum()) > 0
    whole = w.clone()
    dead[0] = NAN
    w.zero_()
    cache.weigh(0, seqs, qh, dead, w)
    assert torch.equal(w[0, 1], whole[0, 1])
    assert torch.isnan(w[0, 0, :, :31]).all() and not torch.isnan(w[0, 0, :, 31:]).any()
    dead[0] = INF
    w.zero_()
    cache.weigh(0, seqs, qh, dead, w)
    assert torch.equal(w, whole)


def test_weights_of_a_call_add_up_to_its_rows():
    """Each row's probabilities sum to one, with the kernels' own lse."""
    b = Batch("bf16", 8, 2, 128, 16, [3, 80, 1], [200, 333, 64], seed=8)
    cache, seqs, q, _, _ = b.cuda()
    lse = torch.empty(b.N, b.heads, device="cuda")
    cache.attend(0, seqs, q, lse=lse)
    w = cache.new_weights(seqs)
    cache.weigh(0, seqs, q, lse, w)
    total = w[0].double().sum(-1).cpu()
    rows = torch.tensor(b.q, dtype=torch.float64)[:, None] * (b.heads // b.kv_heads)
    # cr_attend's sums are of probabilities rounded to bf16 where it rounds them
    assert ((total - rows).abs() <= rows * 2.0 ** -8).all()


def test_weigh_many_ragged_sequences():
    """More sequences than travel with a launch, some without queries or keys."""
    rng = np.random.default_rng(3)
    q = rng.integers(0, 4, 150).tolist()
    lens = [a + int(x) for a, x in zip(q, rng.integers(0, 60, 150))]
    b = Batch("bf16", 4, 2, 32, 4, q, lens, seed=1)
    _weigh_case(b, 0)
    q[7] = 70                                            # ... and a prompt among them
    lens[7] = 90
    _weigh_case(Batch("bf16", 4, 1, 32, 4, q, lens, seed=1), 0)


# rows that go through LDS: more than 512 in a sequence, or some over many tiles
WIDE = {
    "long": dict(dtype="bf16", heads=8, kv_heads=2, d=128, bs=16, q=[133, 0, 3], lens=[300, 4, 100]),
    "long-odd": dict(dtype="bf16", heads=7, kv_heads=1, d=64, bs=8, q=[75, 1], lens=[170, 400]),
    "long-f32": dict(dtype="f32", heads=9, kv_heads=1, d=96, bs=2, q=[60, 2], lens=[60, 300]),
    "many": dict(dtype="bf16", heads=24, kv_heads=8, d=64, bs=32, q=[7, 0, 1, 6] * 10,
                 lens=[150, 40, 1, 190] * 10),
    "many-f32": dict(dtype="f32", heads=12, kv_heads=6, d=32, bs=16, q=[9, 1, 13] * 15,
                     lens=[9, 130, 141] * 15),
}


@pytest.mark.parametrize("name", WIDE)
@pytest.mark.parametrize("kind", ["causal", "intervals", "cap", "slopes", "all"])
def test_weigh_rows_through_lds(name, kind):
    b = Batch(L=1, seed=7 + len(name), fill=-6.0, **WIDE[name])
    rng = np.random.default_rng(6)
    o = {}
    if kind in ("intervals", "all"):
        lo = rng.integers(-5, 180, b.N)
        o.update(lo=lo.tolist(), hi=(lo + rng.integers(-3, 200, b.N)).tolist())
    if kind in ("cap", "all"):
        o["softcap"] = 3.0
    if kind in ("slopes", "all"):
        o.update(slopes=[0.2 * 2.0 ** -(h % 8) for h in range(b.heads)], scale=0.15)
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 0, **o)
    from paper_2609_35139_amd import binding as B
    assert B.cr_weigh_workspace_bytes(cache.layout, seqs.struct, b.heads) > 0
    again = prior.cuda()
    cache.weigh(0, seqs, q, lse, again, **k)
    assert torch.equal(again, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", range(32, 257, 32))
def test_weigh_rows_through_lds_of_every_head_dim(dtype, d):
    _weigh_case(Batch(dtype, 8, 1, d, 16, [70], [170], seed=d), 0)


def test_weigh_rows_through_lds_do_not_look_at_hidden_keys():
    b = Batch("bf16", 8, 1, 64, 16, [80], [150], seed=2, fill=NAN)
    for j in range(40, 150):
        blk, r = b.row(0, j)
        b.pool[0, 0, blk, r] = [INF, -INF, NAN][j % 3]
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 0, hi=[40] * 80)
    blk, r = b.row(0, 3)
    cache.pool[0, 0, blk, r] = NAN
    w2 = prior.cuda()
    cache.weigh(0, seqs, q, lse, w2, **k)
    assert torch.isnan(w2).nonzero().tolist() == [[0, 0, 0, 3]]


@pytest.mark.parametrize("lse_of_one", [NAN, INF])
def test_weigh_rows_through_lds_without_a_sum(lse_of_one):
    """Rows whose lse is -inf, NaN or +inf among more than 512."""
    q = 140
    b = Batch("bf16", 4, 1, 64, 16, [q, q], [q + 30, q + 50], seed=q)
    _, lse, _, _ = attend_oracle(b, 0)
    cache, seqs, qh, _, _ = b.cuda()
    dead = lse.float().cuda()
    dead[:q] = -INF
    w = cache.new_weights(seqs)
    cache.weigh(0, seqs, qh, dead, w)
    assert torch.equal(w[0, 0], torch.zeros_like(w[0, 0])) and float(w[0, 1].sum()) > 0
    whole = w.clone()
    dead[0] = lse_of_one
    w.zero_()
    cache.weigh(0, seqs, qh, dead, w)
    assert torch.equal(w[0, 1], whole[0, 1])
    if lse_of_one == INF:
        assert torch.equal(w, whole)
    else:
        assert torch.isnan(w[0, 0, :, :31]).all() and not torch.isnan(w[0, 0, :, 31:]).any()


def test_weigh_parts_of_few_tiles():
    """One long prompt over a short cache: its rows are split and joined."""
    b = Batch("bf16", 16, 1, 64, 16, [120], [120], seed=6)
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 0)
    for _ in range(2):
        again = prior.cuda()
        cache.weigh(0, seqs, q, lse, again)
        assert torch.equal(again, w)


def test_weigh_strides_pools_and_streams():
    """Queries and weights with gaps, a pool whose heads lie apart, another stream."""
    b = Batch("bf16", 4, 2, 64, 8, [1, 30], [50, 70], L=2, seed=4)
    w, cache, seqs, q, lse, prior, k = _weigh_case(b, 1)
    from paper_2609_35139_amd.serving import PagedCache
    pool = cache.pool.permute(4, 0, 1, 2, 3, 5).contiguous().permute(1, 2, 3, 4, 0, 5)
    other = PagedCache(pool)
    seqs2 = other.sequences(seqs.block_table, seqs.kv_lens, b.off)
    wide = torch.zeros(b.N, 2 * b.heads + 1, b.d + 8, dtype=torch.bfloat16, device="cuda")
    rows = wide[:, 1::2, :b.d]
    rows.copy_(q)
    gaps = torch.full((2, 5, 2, prior.shape[3] + 3), 4.0, device="cuda")
    view = gaps[:, 1::2, :, 1:1 + prior.shape[3]]
    view.copy_(prior)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other.weigh(1, seqs2, rows, lse, view, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(view, w)
    view.fill_(4.0)
    assert torch.equal(gaps, torch.full_like(gaps, 4.0))


def test_weights_and_blocks_past_32_bits():
    """Blocks, rows of weights and lists further than 2^32 elements from their beginning."""
    b = Batch("bf16", 2, 1, 64, 16, [1, 1], [100, 40], seed=3)
    far = 2 * (1 << 21)                                  # blocks of 1,024 elements: 2^32 of them
    pool = torch.empty(1, 2, far + b.n_blocks, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
    pool[:, :, far:] = b.pool.cuda()
    from paper_2609_35139_amd.serving import PagedCache
    cache = PagedCache(pool)
    table = torch.where(b.table >= 0, b.table + far, b.table).cuda()
    lens = _i32(b.lens)
    seqs = cache.sequences(table, lens)
    _, lse, _, _ = attend_oracle(b, 0)
    lse = lse.float()
    width = table.shape[1] * 16
    prior = torch.rand(1, 2, 1, width)
    ref, tol = weigh_oracle(b, 0, lse, prior)
    store = torch.empty((1 << 32) + 2 * width, device="cuda")
    w = torch.as_strided(store, (1, 2, 1, width), (0, 1 << 32, width, 1))
    w.copy_(prior)
    cache.weigh(0, seqs, b.qh.cuda(), lse.cuda(), w)
    assert_within(w, ref, tol, "weights")
    kept, kept_lens = cache.choose(seqs, w, 20, first=1, recent=3)
    k_ref, l_ref = choose_oracle(w.cpu(), b.lens, width, 20, 1, 3)
    assert np.array_equal(kept.cpu().numpy(), k_ref) and np.array_equal(kept_lens.cpu().numpy(), l_ref)
    want, w_ref = compact_oracle(b.pool, b.table, b.lens, k_ref, l_ref, w.cpu())
    cache.compact(seqs, kept, kept_lens, weights=w)
    assert torch.equal(pool[:, :, far:].cpu(), want) and torch.equal(w.cpu(), w_ref)


# ------------------------------------------------------------------- choose
def _layout_cache(L, H, blocks=4, bs=16, dtype=torch.bfloat16, d=32):
    from paper_2609_35139_amd.serving import PagedCache
    return PagedCache(torch.zeros(L, 2, blocks, bs, H, d, dtype=dtype, device="cuda"))


def _choose_case(weights, lens, budget, first=0, recent=0, budgets=None, bs=16):
    L, S, H, slots = weights.shape
    cache = _layout_cache(L, H, bs=bs)
    seqs = cache.sequences(_i32(np.zeros((S, slots // bs))), _i32(lens))
    kept, kept_lens = cache.choose(seqs, weights.cuda(), budget, first=first, recent=recent,
                                   budgets=None if budgets is None else _i32(budgets))
    ref, ref_lens = choose_oracle(weights, lens, slots, budget, first, recent, budgets)
    assert np.array_equal(kept_lens.cpu().numpy(), ref_lens)
    got = kept.cpu().numpy()
    assert np.array_equal(got, ref), np.argwhere(got != ref)[:5]


@pytest.mark.parametrize("slots", [16, 400, 4096, 8192, 20000, 32768, 33008, 70000])
def test_choose_sizes(slots):
    """Every variant: registers of 256 and 512 threads, rows read again."""
    g = torch.Generator().manual_seed(slots)
    w = torch.randn(2, 3, 1, slots, generator=g).mul(2).exp()
    w[torch.rand(w.shape, generator=g) < 0.2] = 0.0
    w[torch.rand(w.shape, generator=g) < 0.1] = 0.125
    _choose_case(w, [slots, slots - 7, slots // 3], max(1, slots // 3 - 1), 4, 9)


@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (1, 5, 5), (50, 0, 50), (50, 50, 0),
                                                 (50, 20, 40), (63, 1, 1), (64, 0, 0), (65, 9, 9), (500, 3, 3)])
def test_choose_budgets(budget, first, recent):
    w = torch.rand(1, 5, 2, 64, generator=torch.Generator().manual_seed(budget))
    _choose_case(w, [64, 63, 0, 1, 200], budget, first, recent)
    _choose_case(w, [64, 50, -3, 64, 64], budget, first, recent, budgets=[budget, 10, 5, 0, -4])


@pytest.mark.parametrize("values", ["equal", "two", "infinite", "nan", "negative", "denormal", "huge", "steps"])
@pytest.mark.parametrize("slots", [96, 5008])
def test_choose_values(values, slots):
    g = torch.Generator().manual_seed(len(values))
    r = torch.rand(1, 2, 2, slots, generator=g)
    w = {"equal": torch.full_like(r, 0.3), "two": (r > 0.5).float(),
         "infinite": torch.where(r < 0.3, torch.full_like(r, INF), torch.where(r < 0.4, torch.full_like(r, -INF), r)),
         "nan": torch.where(r < 0.6, torch.full_like(r, NAN), torch.where(r < 0.7, torch.full_like(r, -INF), -r)),
         "negative": torch.where(r < 0.2, torch.zeros_like(r), torch.where(r < 0.4, -torch.zeros_like(r), r - 0.6)),
         "denormal": (r * 40).floor() * 2.0 ** -149, "huge": torch.where(r < 0.5, -r, r) * 3e38,
         "steps": torch.nextafter(torch.ones_like(r), torch.where(r < 0.5, torch.zeros_like(r), 2 + r))}[values]
    _choose_case(w, [slots, slots - 5], slots // 2, 3, 10)


def test_choose_rows_that_begin_anywhere_and_many_heads():
    w = torch.rand(2, 2, 3, 8 * 11, generator=torch.Generator().manual_seed(1))
    store = torch.zeros(2, 2, 3, 8 * 11 + 5).cuda()
    cache = _layout_cache(2, 3, bs=8)
    seqs = cache.sequences(_i32(np.zeros((2, 11))), _i32([88, 70]))
    view = store[..., 3:91]
    view.copy_(w)
    kept, lens = cache.choose(seqs, view, 33, first=2, recent=5)
    ref, ref_lens = choose_oracle(w, [88, 70], 88, 33, 2, 5)
    assert np.array_equal(kept.cpu().numpy(), ref) and np.array_equal(lens.cpu().numpy(), ref_lens)
    mine, my_lens = torch.empty_like(kept), torch.empty_like(lens)
    assert cache.choose(seqs, view, 33, first=2, recent=5, kept=mine, kept_lens=my_lens) == (mine, my_lens)
    assert torch.equal(mine, kept) and torch.equal(my_lens, lens)


# ------------------------------------------------------------------ compact
def _compact_case(dtype="bf16", L=2, H=2, d=64, bs=8, lens=(60, 33, 5), budget=24, moved=False,
                  weights=True, kept=None, change=None, seed=0):
    b = Batch(dtype, H, H, d, bs, [0] * len(lens), list(lens), L=L, seed=seed, table_slack=1)
    rng = np.random.default_rng(seed)
    S = len(lens)
    if kept is None:
        kept = np.full((L, S, H, budget), -1, dtype=np.int32)
        for l in range(L):
            for s in range(S):
                for h in range(H):
                    m = min(budget, max(lens[s], 0))
                    kept[l, s, h, :m] = np.sort(rng.permutation(max(lens[s], 0))[:m])
    kept_lens = np.array([min(max(n, 0), budget) for n in lens], dtype=np.int32)
    out = None
    if moved:
        blocks = -(-budget // bs)
        fresh = torch.randn(L, 2, S * blocks, bs, H, d).to(TORCH[dtype])
        b.pool = torch.cat([b.pool, fresh], 2)
        out = torch.tensor(rng.permutation(S * blocks).reshape(S, blocks) + b.n_blocks, dtype=torch.int32)
        b.n_blocks += S * blocks
    if change:
        kept, kept_lens, out = change(b, kept, kept_lens, out)
    w = torch.rand(L, S, H, b.table.shape[1] * bs) if weights else None
    want, w_ref = compact_oracle(b.pool, b.table, b.lens, kept, kept_lens, w, out)
    cache, seqs, _, _, _ = b.cuda()
    w_dev = None if w is None else w.cuda()
    cache.compact(seqs, _i32(kept), _i32(kept_lens), weights=w_dev,
                  block_table=None if out is None else out.cuda())
    assert torch.equal(cache.pool.cpu(), want)
    if weights:
        assert torch.equal(w_dev.cpu(), w_ref)


@pytest.mark.parametrize("moved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 224, 256])
def test_compact_rows_of_every_size(d, dtype, moved):
    _compact_case(dtype, d=d, moved=moved, seed=d)


@pytest.mark.parametrize("moved", [False, True])
@pytest.mark.parametrize("bs", [1, 16, 256])
def test_compact_many_steps(bs, moved):
    """Lists of several steps, whole ones and ragged ones, identities among them."""
    _compact_case(L=1, H=2, d=128, bs=bs, lens=(1500, 700, 1, 0), budget=650, moved=moved, seed=bs)
    keep = np.arange(650, dtype=np.int32)[None, None, None].repeat(2, 1).repeat(2, 2)
    keep = np.ascontiguousarray(keep)
    keep[0, 0, 0, 300:] += 400
    _compact_case(L=1, H=2, d=128, bs=bs, lens=(1500, 700), budget=650, moved=moved, kept=keep)


def test_compact_many_workgroups_and_few():
    _compact_case(L=9, H=8, d=64, bs=16, lens=(200, 90, 64, 201), budget=70, seed=4)
    _compact_case(L=1, H=1, d=256, dtype="f32", bs=16, lens=(900,), budget=300, seed=5)


@pytest.mark.parametrize("moved", [False, True])
def test_compact_entries_that_are_none(moved):
    """Slots outside the sequence, blocks that are none, lengths outside the list: nothing moves."""
    def change(b, kept, kept_lens, out):
        kept = np.full_like(kept, -1)
        kept[..., :6] = [-7, 2, 5, 1 << 30, 11, 13]
        b.table[1, 0] = -1
        if out is not None:
            out[0, 0] = b.n_blocks + 5
            out = out[:, :2].contiguous()                # ... and a table shorter than the list
        return kept, np.array([6, 1 << 30, -2], dtype=np.int32), out
    _compact_case(moved=moved, change=change, seed=2)


def test_compact_without_weights_and_of_odd_strides():
    _compact_case(weights=False)
    b = Batch("bf16", 3, 3, 64, 8, [0, 0], [40, 25], L=2, seed=7)
    from paper_2609_35139_amd.serving import PagedCache
    pool = b.pool.cuda().permute(4, 2, 0, 1, 3, 5).contiguous().permute(2, 3, 1, 4, 0, 5)
    cache = PagedCache(pool)
    seqs = cache.sequences(b.table.cuda(), _i32(b.lens))
    w = torch.rand(2, 2, 3, b.table.shape[1] * 8)
    kept, lens = choose_oracle(w, b.lens, w.shape[3], 16, 1, 2)
    want, _ = compact_oracle(b.pool, b.table, b.lens, kept, lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    cache.compact(seqs, _i32(kept), _i32(lens), stream=s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.equal(pool.cpu(), want)


# ------------------------------------------------------------------- sample
def _logits(R, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, V, generator=g) * spread
    n = min(V, 40)
    at = torch.randint(0, V, (R, n), generator=g)
    x.scatter_add_(1, at, torch.empty(R, n).exponential_(generator=g) * 2 + 3 * spread)
    return x.to(TORCH[dtype])


def _sample_case(x, u=None, seed=0, **k):
    from paper_2609_35139_amd.serving import sample
    if u is None:
        u = torch.rand(x.shape[0], generator=torch.Generator().manual_seed(seed))
    dev = {n: v.cuda() if isinstance(v, torch.Tensor) else v for n, v in k.items()}
    tokens, log_p = sample(x.cuda(), u.cuda(), **dev)
    ref, ref_p = sample_oracle(x, u, **k)
    got = tokens.cpu().numpy()
    assert np.array_equal(got, ref), (np.argwhere(got != ref)[:5], got[:8], ref[:8])
    p = log_p.double().cpu().numpy()
    dead = ref < 0
    assert (p[dead] == -np.inf).all()
    p, ref_p = p[~dead], ref_p[~dead]
    assert (np.abs(p - ref_p) <= log_prob_bound(ref_p, x.shape[1])).all()
    return tokens, log_p


SETTINGS = [dict(), dict(temperature=0.0), dict(top_k=1), dict(top_k=20, top_p=0.8, temperature=0.7),
            dict(top_k=200), dict(top_k=1500, top_p=0.9), dict(top_p=0.9), dict(top_p=0.5, temperature=0.3),
            dict(min_p=0.05), dict(min_p=1.0), dict(top_p=0.99, min_p=0.001, temperature=1.5),
            dict(top_k=7000, min_p=0.01), dict(temperature=50.0, top_p=0.6), dict(temperature=1e-3)]


@pytest.mark.parametrize("k", SETTINGS, ids=lambda k: ",".join(f"{a}={b}" for a, b in k.items()) or "plain")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 5, 17, 1000, 2049, 9001, 40000])
def test_sample(V, dtype, k):
    _sample_case(_logits(9, V, dtype, V), seed=V, **k)


@pytest.mark.parametrize("dtype,V", [("bf16", 151936), ("f32", 128256), ("f32", 300001), ("bf16", 1 << 19)])
def test_sample_large_vocabularies(dtype, V):
    x = _logits(6, V, dtype, 3)
    flat = _logits(6, V, dtype, 4, spread=0.5)
    for k in (dict(), dict(top_p=0.95), dict(top_k=50, top_p=0.9), dict(top_k=V // 3, top_p=0.8), dict(min_p=0.02)):
        _sample_case(x, seed=1, **k)
        _sample_case(flat, seed=2, **k)


def test_sample_settings_of_every_row():
    R = 64
    rng = np.random.default_rng(4)
    pick = lambda v, dtype: torch.tensor(rng.choice(v, R), dtype=dtype)     # noqa: E731
    k = dict(temperature=pick([0.0, -1.0, NAN, 0.3, 1.0, 2.0, INF], torch.float32),
             top_k=pick([-5, 0, 1, 2, 30, 700, 1 << 30], torch.int32),
             top_p=pick([1.0, 2.0, 0.9, 0.3, 0.0, -1.0, NAN], torch.float32),
             min_p=pick([0.0, -1.0, 0.1, 1.0, 1.5, NAN], torch.float32))
    for V in (900, 5000):
        _sample_case(_logits(R, V, "f32", V), **k)
        _sample_case(_logits(R, V, "bf16", V), **k)


@pytest.mark.parametrize("V", [300, 6000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_equal_logits(V, dtype):
    """Equal ones count by their index, in lists and in bins that hold nothing else."""
    u = torch.tensor([0.0, 0.25, 0.5, 0.999, 1.0])
    x = torch.full((5, V), 1.25).to(TORCH[dtype])
    for k in (dict(), dict(top_k=40), dict(top_k=V - 1), dict(top_p=0.25), dict(top_k=V // 2, top_p=0.5),
              dict(min_p=0.5), dict(temperature=0.0)):
        _sample_case(x, u, **k)
    x[:, ::3] = 1.0                                       # two values, thousands of each
    x[:, 1::3] = -2.0
    for k in (dict(), dict(top_k=V // 2), dict(top_p=0.9), dict(top_k=V // 3 + 5, top_p=0.95)):
        _sample_case(x, u, **k)


@pytest.mark.parametrize("V", [200, 6000])
def test_sample_values_that_are_not_numbers(V):
    x = _logits(8, V, "f32", 5)
    x[0] = -INF
    x[1] = NAN
    x[2, ::2] = -INF
    x[3, ::3] = NAN
    x[4, [5, 50, 60]] = INF
    x[5] = -3.4028234663852886e38                         # the type's lowest, one ordinary one
    x[5, 77] = 1.0
    x[6, : V // 2] = -3.4028234663852886e38
    x[7] = 3.4028234663852886e38
    x[7, 3] = -3.4028234663852886e38
    for k in (dict(), dict(top_k=2), dict(top_p=0.7), dict(top_k=V // 2, top_p=0.9), dict(min_p=0.2),
              dict(temperature=0.0), dict(temperature=1e-30), dict(temperature=INF)):
        _sample_case(x, **k)
        _sample_case(x.to(torch.bfloat16), **k)


@pytest.mark.parametrize("V", [500, 7000])
def test_sample_far_from_zero_and_close_together(V):
    """Logits whose differences are their last bits, and denormal ones."""
    r = torch.rand(4, V, generator=torch.Generator().manual_seed(V))
    for x in (1e6 + (r * 64).floor() / 16, -1e30 * (1 + (r * 4).floor() * 2.0 ** -22),
              (r * 3000).floor() * 2.0 ** -149, 1 + (r * 9000).floor() * 2.0 ** -23):
        for k in (dict(), dict(top_p=0.5), dict(top_k=300), dict(top_k=V // 2, top_p=0.5),
                  dict(temperature=1e-3, top_p=0.9), dict(min_p=0.9)):
            _sample_case(x.float(), **k)


def test_sample_random_numbers_at_their_ends():
    x = _logits(8, 5000, "f32", 1)
    u = torch.tensor([0.0, -0.5, 1.0, 7.0, NAN, INF, 1 - 2.0 ** -24, 2.0 ** -149])
    for k in (dict(), dict(top_k=10), dict(top_p=0.9)):
        ref_u = torch.nan_to_num(u, nan=0.0, posinf=2.0)
        from paper_2609_35139_amd.serving import sample
        tokens, _ = sample(x.cuda(), u.cuda(), **k)
        ref, _ = sample_oracle(x, ref_u, **k)
        assert np.array_equal(tokens.cpu().numpy(), ref)


@pytest.mark.parametrize("V", [1, 700, 9000, 40000])
def test_sample_of_one_token_that_stays(V):
    """Alone, a token's probability is 1 and its log exactly 0, whatever the logits are."""
    from paper_2609_35139_amd.serving import sample
    x = _logits(64, V, "f32", V + 1)
    x[torch.arange(64), x.argmax(1)] += 20
    u = torch.rand(64, generator=torch.Generator().manual_seed(V))
    for k in (dict(top_p=0.5, temperature=0.33), dict(top_p=0.5, top_k=V // 3), dict(min_p=0.9), dict(top_k=1)):
        tokens, log_p = sample(x.cuda(), u.cuda(), **k)
        assert torch.equal(tokens.cpu().long(), x.argmax(1))
        assert torch.equal(log_p.cpu(), torch.zeros(64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_rows_anywhere_and_outputs_given(dtype):
    """Rows that begin on any element, further apart than they are long; one row of all."""
    x = _logits(7, 3001, dtype, 2)
    store = torch.full((7, 3010), 50.0, dtype=TORCH[dtype], device="cuda")   # larger than any logit
    store[:, 3:3004] = x.cuda()
    from paper_2609_35139_amd.serving import sample
    u = torch.rand(7, generator=torch.Generator().manual_seed(0))
    tokens = torch.full((9,), -9, dtype=torch.int32, device="cuda")
    log_p = torch.full((9,), -9.0, device="cuda")
    for k in (dict(), dict(top_k=9), dict(top_p=0.8), dict(temperature=0.0)):
        got = sample(store[:, 3:3004], u.cuda(), tokens=tokens[1:8], log_probs=log_p[1:8], **k)
        ref, _ = sample_oracle(x, u, **k)
        assert np.array_equal(got[0].cpu().numpy(), ref)
        assert tokens[0] == tokens[8] == -9 and log_p[0] == log_p[8] == -9
    one = x[:1].cuda().expand(7, -1)                     # stride 0
    got, _ = sample(one, u.cuda(), top_p=0.9)
    ref, _ = sample_oracle(x[:1].expand(7, -1), u, top_p=0.9)
    assert np.array_equal(got.cpu().numpy(), ref)


def test_sample_follows_the_probabilities():
    """65,536 draws of one row: every token's share within five standard deviations."""
    x = torch.tensor([[0.0, 1.0, -1.0, 2.0, 0.5, -3.0]])
    n = 1 << 16
    from paper_2609_35139_amd.serving import sample
    u = torch.rand(n, generator=torch.Generator().manual_seed(2)).cuda()
    tokens, _ = sample(x.cuda().expand(n, -1), u, temperature=0.8)
    p = torch.softmax(x[0].double() / 0.8, 0)
    share = torch.bincount(tokens.cpu().long(), minlength=6).double() / n
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()


# ----------------------------------------------------------------- together
def test_an_answer_within_a_budget():
    """A prompt, then steps that append, attend, weigh and sample; whenever the cache is over
    its budget the slots are chosen and compacted.  Every part against its oracle, on the cache
    as it is by then."""
    from paper_2609_35139_amd.serving import PagedCache, sample
    L, heads, H, d, bs, V, blocks = 2, 4, 2, 64, 8, 500, 8
    g = torch.Generator().manual_seed(1)
    S = 2
    b = Batch("bf16", heads, H, d, bs, [30, 21], [30, 21], L=L, seed=1, table_slack=4, spare=10)
    ids = torch.randperm(b.n_blocks, generator=g)[:S * b.table.shape[1]].reshape(S, -1).int()
    b.table = ids
    cache = PagedCache(b.pool.cuda())
    table, lens = b.table.cuda(), _i32(b.lens)
    budget, head = 24, torch.randn(d * heads, V, generator=g).cuda() * 0.05
    position = torch.tensor(b.lens)
    weights = None
    for step in range(6):
        q = [30, 21] if step == 0 else [1, 1]
        off = np.concatenate([[0], np.cumsum(q)])
        seqs = cache.sequences(table, lens, off)
        weights = cache.new_weights(seqs) if weights is None else weights
        new = torch.randn(sum(q), heads + 2 * H, d, generator=g).to(torch.bfloat16)
        pos = torch.cat([torch.arange(p - n, p) for p, n in zip(position.tolist(), q)])
        for layer in range(L):
            dev = new.cuda()
            rot = cache.append(layer, seqs, dev[:, heads:heads + H], dev[:, heads + H:], q=dev[:, :heads],
                               rope=dict(theta=1e4), positions=pos.int().cuda())
            b.pool, b.q, b.lens, b.N, b.off = cache.pool.cpu(), q, lens.tolist(), sum(q), off
            b.qh = rot.cpu()
            lse = torch.empty(sum(q), heads, device="cuda")
            before = weights.cpu()
            out = cache.attend(layer, seqs, rot, lse=lse)
            cache.weigh(layer, seqs, rot, lse, weights)
            ref, ref_lse, tol, _ = attend_oracle(b, layer)
            assert_within(out, ref, tol, "attention")
            ref, tol = weigh_oracle(b, layer, lse.cpu(), before)
            assert_within(weights, ref, tol, "weights")
        last = out[torch.tensor(np.cumsum(q) - 1)].float().reshape(S, -1) @ head
        u = torch.rand(S, generator=g)
        tokens, _ = sample(last, u.cuda(), temperature=0.8, top_k=40, top_p=0.9)
        ref, _ = sample_oracle(last.cpu(), u, temperature=0.8, top_k=40, top_p=0.9)
        assert np.array_equal(tokens.cpu().numpy(), ref)
        if max(lens.tolist()) > budget:
            kept, kept_lens = cache.choose(seqs, weights, budget, first=2, recent=6)
            k_ref, l_ref = choose_oracle(weights.cpu(), lens.tolist(), weights.shape[3], budget, 2, 6)
            assert np.array_equal(kept.cpu().numpy(), k_ref)
            want, w_ref = compact_oracle(cache.pool.cpu(), b.table, lens.tolist(), k_ref, l_ref, weights.cpu())
            cache.compact(seqs, kept, kept_lens, weights=weights)
            assert torch.equal(cache.pool.cpu(), want) and torch.equal(weights.cpu(), w_ref)
            lens.copy_(kept_lens)
        lens += 1
        position += 1


def test_steps_in_a_captured_graph_on_another_stream():
    """Attend, weigh, choose, compact and sample captured once and replayed as lengths and
    logits change, against the eager calls, with eager work in between."""
    from paper_2609_35139_amd.serving import PagedCache, sample
    b = Batch("bf16", 8, 2, 64, 8, [1, 1, 1], [60, 45, 64], L=2, seed=5)
    table, lens = b.table.cuda(), _i32(b.lens)
    x = _logits(3, 6000, "f32", 1).cuda()
    u = torch.rand(3, generator=torch.Generator().manual_seed(3)).cuda()
    q = b.qh.cuda()

    def make():
        cache = PagedCache(b.pool.cuda())
        seqs = cache.sequences(table, lens)
        return dict(cache=cache, seqs=seqs, w=cache.new_weights(seqs), lse=torch.empty(3, 8, device="cuda"),
                    out=torch.empty_like(q), kept=torch.empty(2, 3, 2, 20, dtype=torch.int32, device="cuda"),
                    lens=torch.empty(3, dtype=torch.int32, device="cuda"),
                    t=torch.empty(3, dtype=torch.int32, device="cuda"), p=torch.empty(3, device="cuda"))

    def step(z, ws, stream=None):
        c = z["cache"]
        for layer in range(2):
            c.attend(layer, z["seqs"], q, out=z["out"], lse=z["lse"], workspace=ws, stream=stream)
            c.weigh(layer, z["seqs"], q, z["lse"], z["w"], stream=stream)
        c.choose(z["seqs"], z["w"], 20, first=1, recent=4, kept=z["kept"], kept_lens=z["lens"], stream=stream)
        c.compact(z["seqs"], z["kept"], z["lens"], weights=z["w"], stream=stream)
        sample(x, u, top_p=0.9, tokens=z["t"], log_probs=z["p"], stream=stream)

    eager, graphed = make(), make()
    ws_e, ws_g = (z["cache"].workspace(z["seqs"], 8) for z in (eager, graphed))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(graphed, ws_g, s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(graphed, ws_g, s)
    torch.cuda.synchronize()
    graphed["cache"].pool.copy_(b.pool)
    graphed["w"].zero_()
    for n in ([60, 45, 64], [31, 64, 0], [64, 1, 33], [20, 25, 60]):
        lens.copy_(_i32(n))
        x.add_(torch.randn(x.shape, generator=torch.Generator().manual_seed(sum(n))).cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(eager, ws_e)
        torch.cuda.synchronize()
        for name in ("w", "out", "kept", "lens", "t", "p"):
            assert torch.equal(eager[name], graphed[name]), name
        assert torch.equal(eager["cache"].pool, graphed["cache"].pool)
        _ = (x * 2).sum().item()


def test_weigh_replays_with_a_workspace_of_its_own():
    """A captured prompt call beside an eager one of the same cache on another stream."""
    b = Batch("bf16", 8, 1, 64, 16, [90], [150], seed=2)
    cache, seqs, q, _, _ = b.cuda()
    lse = torch.empty(b.N, 8, device="cuda")
    cache.attend(0, seqs, q, lse=lse)
    from paper_2609_35139_amd import binding as B
    need = B.cr_weigh_workspace_bytes(cache.layout, seqs.struct, 8)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    ref = cache.weigh(0, seqs, q, lse, cache.new_weights(seqs))
    w = cache.new_weights(seqs)
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    cache.weigh(0, seqs, q, lse, w, workspace=ws, stream=s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        cache.weigh(0, seqs, q, lse, w, workspace=ws, stream=s)
    for _ in range(3):
        w.zero_()
        w2 = cache.new_weights(seqs)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        cache.weigh(0, seqs, q, lse, w2, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(w, ref) and torch.equal(w2, ref)


def test_refusals_of_the_torch_side():
    b = Batch("bf16", 4, 2, 64, 8, [1, 1], [20, 30], seed=1)
    cache, seqs, q, _, _ = b.cuda()
    lse = torch.zeros(2, 4, device="cuda")
    w = cache.new_weights(seqs)
    for bad in (w.double(), w.cpu()):
        with pytest.raises(TypeError):
            cache.weigh(0, seqs, q, lse, bad)
    for bad in (w[..., :-1], w[:, :1], w.transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(ValueError):
            cache.weigh(0, seqs, q, lse, bad)
    with pytest.raises(TypeError):
        cache.weigh(0, seqs, q, lse[:1], w)
    with pytest.raises(ValueError):
        cache.weigh(0, Batch("bf16", 4, 2, 64, 8, [1], [9], seed=1).cuda()[1], q, lse, w)
    kept, lens = cache.choose(seqs, w, 8)
    for bad in (kept.long(), kept[..., ::2], kept[:, :1]):
        with pytest.raises(TypeError):
            cache.compact(seqs, bad, lens)
    with pytest.raises(TypeError):
        cache.compact(seqs, kept, lens, block_table=seqs.block_table[:1])
    with pytest.raises(TypeError):
        cache.choose(seqs, w, 8, budgets=torch.zeros(3, dtype=torch.int32, device="cuda"))
    from paper_2609_35139_amd.serving import sample
    x, u = torch.zeros(3, 50, device="cuda"), torch.zeros(3, device="cuda")
    for kw in (dict(u=u[:2]), dict(u=u.double()), dict(temperature=torch.zeros(2, device="cuda")),
               dict(top_k=torch.zeros(3, device="cuda")), dict(tokens=torch.zeros(3, device="cuda"))):
        with pytest.raises(TypeError):
            sample(x, kw.pop("u", u), **kw)
    with pytest.raises(TypeError):
        sample(x.half(), u)
    with pytest.raises(ValueError):
        sample(x.t(), torch.zeros(50, device="cuda"))
    assert sample(x[:0], u[:0])[0].shape == (0,)


def test_profile_names_the_launches():
    from paper_2609_35139_amd import binding as B
    from paper_2609_35139_amd.serving import sample
    b = Batch("bf16", 4, 2, 64, 8, [1, 1], [20, 30], seed=1)
    cache, seqs, q, _, _ = b.cuda()
    lse, w = torch.empty(2, 4, device="cuda"), cache.new_weights(seqs)
    cache.attend(0, seqs, q, lse=lse)
    torch.cuda.synchronize()
    B.cr_profile_enable(16)
    try:
        cache.weigh(0, seqs, q, lse, w)
        kept, lens = cache.choose(seqs, w, 8)
        cache.compact(seqs, kept, lens, weights=w)
        sample(torch.zeros(2, 100, device="cuda"), torch.zeros(2, device="cuda"))
        names = [x["name"] for x in B.cr_profile_read()]
    finally:
        B.cr_profile_enable(0)
    assert names == ["weigh_keys", "choose_slots", "compact_kv", "sample"]
