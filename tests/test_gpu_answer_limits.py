"""Calls of cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample at the
limits of their ranges, on the GPU."""
import math

import numpy as np
import pytest
import torch

from serving_helpers import TORCH, Batch
from test_gpu_answer import _i32, _layout_cache, _sample_case, _weigh_case

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35139_amd import binding
    binding.load()


# -------------------------------------------------------------------- weigh
def _again(case, b, **o):
    """The oracle's weights, and the same bits from a second call."""
    w, cache, seqs, q, lse, prior, k = case
    again = prior.cuda()
    cache.weigh(0, seqs, q, lse, again, **k)
    assert torch.equal(again, w)
    return w, cache, seqs, q, lse, prior, k


# single tokens: (a sequence's queries, slots), more tiles of keys than there are waves, so
# that a wave has a run of tiles that passes from sequence to sequence
RUNS = {"bf16": (32, dict(dtype="bf16", heads=32, kv_heads=16, d=64, bs=16)),
        "f32": (32, dict(dtype="f32", heads=32, kv_heads=16, d=32, bs=8)),
        "f32-wide": (16, dict(dtype="f32", heads=8, kv_heads=8, d=160, bs=64))}


@pytest.mark.parametrize("name", RUNS)
def test_weigh_single_tokens_of_more_tiles_than_waves(name):
    keys, sizes = RUNS[name]                             # keys of a tile
    rng = np.random.default_rng(len(name))
    S, most = 64, 1024
    lens = rng.integers(1, most + 1, S)
    lens[rng.random(S) < 0.15] = 0
    lens[5], lens[6], lens[S - 1] = most, 1, 33
    q = np.minimum(rng.choice([0, 1, 1, 1, 2, 8], S), lens)
    q[5] = 1
    b = Batch(q=q.tolist(), lens=lens.tolist(), seed=2, **sizes)
    assert sum(-(-n // keys) for n, m in zip(lens, q) if m) > 2 * 4 * -(-1024 // sizes["kv_heads"])
    case = _again(_weigh_case(b, 0), b)
    from paper_2609_35139_amd import binding as B
    assert B.cr_weigh_workspace_bytes(case[1].layout, case[2].struct, b.heads) == 0
    lo = rng.integers(0, 500, b.N)
    _weigh_case(b, 0, lo=lo.tolist(), hi=(lo + rng.integers(0, 600, b.N)).tolist(), softcap=3.0,
                slopes=[0.01] * b.heads)


@pytest.mark.parametrize("kv_heads,dtype", [(1, "bf16"), (1, "f32"), (6, "bf16")])
def test_weigh_many_ragged_sequences_with_a_prompt_through_lds(kv_heads, dtype):
    """More sequences than travel with a launch (their offsets in the workspace, beside what the
    rows bring and, for few tiles, the parts), a prompt of more than 512 rows for a KV head among
    them, sequences without queries before, behind and last."""
    rng = np.random.default_rng(3)
    q = rng.integers(0, 4, 150)
    lens = q + rng.integers(0, 60, 150)
    q[7], lens[7] = 140, 150
    q[[6, 8, 9, 148, 149]] = 0
    group = 4
    b = Batch(dtype, group * kv_heads, kv_heads, 32, 4, q.tolist(), lens.tolist(), seed=1)
    case = _again(_weigh_case(b, 0), b)
    from paper_2609_35139_amd import binding as B
    need = B.cr_weigh_workspace_bytes(case[1].layout, case[2].struct, b.heads)
    rows, keys = b.N * b.heads * 32, 128 if dtype == "bf16" else 64          # of a tile
    few = 2 * 150 * kv_heads * -(-b.table.shape[1] * 4 // keys) <= 768       # tiles that share parts
    assert few == (kv_heads == 1 and dtype == "bf16")
    assert rows + 151 * 4 < need < rows + 8192 + 768 * 4 * keys * few
    assert not few or need > rows + 768 * 4 * keys
    lo = rng.integers(-5, 100, b.N)
    _weigh_case(b, 0, lo=lo.tolist(), hi=(lo + rng.integers(-3, 90, b.N)).tolist(), softcap=2.5)


@pytest.mark.parametrize("dtype,lens", [("bf16", [1000] * 16 + [1024, 0, 17]), ("f32", [500] * 16 + [512, 1])])
def test_weigh_through_lds_of_more_units_than_workgroups(dtype, lens):
    """More than 8,192 (tile, KV head) units: a workgroup takes several."""
    q = [min(n, 17) for n in lens]
    b = Batch(dtype, 64, 64, 32, 16, q, lens, seed=4)
    keys = 128 if dtype == "bf16" else 64
    assert sum(-(-n // keys) for n in lens) * 64 > 8192
    case = _again(_weigh_case(b, 0), b)
    from paper_2609_35139_amd import binding as B
    assert B.cr_weigh_workspace_bytes(case[1].layout, case[2].struct, 64) > 0


# rows of a KV head: one instruction's, read where they lie, through LDS (in steps where whole
# queries make up a round of rows, else row by row); heads of a group 1, 4, 5
FAR = [(1, 4, 64), (30, 4, 64), (140, 4, 64), (120, 5, 128), (600, 1, 32), (140, 4, 256)]


@pytest.mark.parametrize("q,group,d", FAR)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weigh_queries_that_lie_apart(q, group, d, dtype):
    """Queries with gaps between tokens and heads; heads further apart than the steps of the rows'
    addresses take; tokens so; and as far as they do take."""
    b = Batch(dtype, group, 1, d, 16, [q], [q + 70], seed=q + d)
    w, cache, seqs, rows, lse, prior, k = _weigh_case(b, 0)
    for token, head in ((group * (d + 16) + 40, d + 16), (d, (1 << 20) + 8), ((1 << 24) + 8, d),
                        ((1 << 23) - 4096, d)):
        n = (q - 1) * token + (group - 1) * head + d
        print(f"strides {token} {head}, {n >> 20} Mi elements", flush=True)
        store = torch.empty(n, dtype=TORCH[dtype], device="cuda")
        if n < 1 << 24:
            store.fill_(NAN)
        apart = torch.as_strided(store, (q, group, d), (token, head, 1))
        apart.copy_(rows)
        again = prior.cuda()
        cache.weigh(0, seqs, apart, lse, again)
        assert torch.equal(again, w)
        del store, apart
        torch.cuda.empty_cache()


# ------------------------------------------------------------------- choose
# 256 threads (more than 512 rows of up to 8,192 slots), 512 (up to 32,768), 1,024
CHOOSE = [(36, 5, 4, 400), (18, 4, 8, 8192), (12, 6, 4, 5008), (3, 20, 6, 20000), (2, 6, 16, 33008)]


@pytest.mark.parametrize("L,S,H,slots", CHOOSE)
@pytest.mark.parametrize("value", [0.0, 0.3, NAN, -INF, INF])
def test_choose_where_nothing_is_larger(L, S, H, slots, value):
    """All weights equal, above all those of a cache that no query has weighed yet: the range of
    the weights is one number, and the lowest slots stay."""
    cache = _layout_cache(L, H)
    lens = [slots - s for s in range(S)]
    seqs = cache.sequences(_i32(np.zeros((S, slots // 16))), _i32(lens))
    w = cache.new_weights(seqs)
    assert not w.any()
    w.fill_(value)
    budget, first, recent = slots // 3, 3, 11
    want = np.empty((S, budget), dtype=np.int32)
    for s, n in enumerate(lens):
        want[s] = np.concatenate([np.arange(budget - recent), np.arange(n - recent, n)])
    want = _i32(want)[None, :, None].expand(L, S, H, budget)
    for _ in range(3):
        kept, kept_lens = cache.choose(seqs, w, budget, first=first, recent=recent)
        assert torch.equal(kept, want)
        assert kept_lens.tolist() == [budget] * S


# ------------------------------------------------------------------- sample
def _close_logits(R, V, dtype, largest, seed):
    """Rows whose largest logits are `largest` and the next floats below it, some of them equal;
    the others lie anywhere down to 0 or twice as far from it."""
    rng = np.random.default_rng(seed)
    bits = 16 if dtype == "bf16" else 0
    a = np.array([abs(largest)], dtype=np.float32).view(np.int32)[0] >> bits
    x = np.empty((R, V), dtype=np.float32)
    for r in range(R):
        away = rng.integers(0, 1 << (23 - bits), V)                    # up to twice, or half, as large
        near = rng.permutation(V)[:min(V, 60)]
        away[near] = np.minimum(rng.geometric(0.3, len(near)) - 1, 12)
        b = (a + away if largest < 0 else a - away).astype(np.int32) << bits
        x[r] = b.view(np.float32) * (-1 if largest < 0 else 1)
    return torch.from_numpy(x).to(TORCH[dtype])


# no filter; top-k by a list of the largest, by bins and of most; top-p; min-p; several
PATHS = [dict(), dict(top_k=20), dict(top_k=1500), dict(top_k=3000, top_p=0.7), dict(top_p=0.9),
         dict(top_p=0.4, min_p=0.01), dict(min_p=0.05), dict(top_k=40, top_p=0.8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 6000, 40000])
@pytest.mark.parametrize("largest,temperature", [
    (20.0, 1e-6), (20.0, 1e-7), (20.0, 1e-8), (-20.0, 1e-8), (9.0, 1e-9), (700.0, 1e-10), (20.0, 1e-12),
    (20.0, 0.01), (-300.0, 0.5), (1e-3, 1e-12), (1e8, 1.0), (-1e9, 1.0), (1.3e9, 1.0), (2e9, 1.0),
    (1e11, 1.0), (-1e12, 1.0), (1e13, 1.0), (1e30, 1e20), (1e4, 1e-4)])
def test_sample_where_the_next_float_weighs_little_or_nothing(largest, temperature, V, dtype):
    """Temperatures of a few last bits of the logits and less: floats below the largest weigh what
    the temperature says, and nothing if they lie too far, in every path."""
    x = _close_logits(5, V, dtype, largest, V)
    for k in PATHS:
        _sample_case(x, seed=3, temperature=temperature, **k)


@pytest.mark.parametrize("V", [900, 20000])
def test_sample_small_temperatures_of_every_row(V):
    R = 48
    rng = np.random.default_rng(V)
    x = torch.cat([_close_logits(R // 4, V, "f32", m, V) for m in (16.5, -700.0, 3e5, 5e9)])
    pick = lambda v, dtype: torch.tensor(rng.choice(v, R), dtype=dtype)     # noqa: E731
    _sample_case(x, temperature=pick([1e-30, 1e-12, 1e-8, 1e-7, 1e-5, 0.02, 1.0], torch.float32),
                 top_k=pick([0, 0, 7, 300, 5000], torch.int32), top_p=pick([1.0, 0.95, 0.5], torch.float32),
                 min_p=pick([0.0, 0.0, 0.1], torch.float32))


def test_sample_one_row_of_a_large_vocabulary_at_small_temperatures():
    for dtype, V in (("bf16", 151936), ("f32", 300001)):
        x = _close_logits(1, V, dtype, 18.0, 4)
        for t in (1e-6, 1e-8, 1e-10):
            for k in (dict(), dict(top_k=50), dict(top_k=9000), dict(top_p=0.9)):
                _sample_case(x, temperature=t, **k)


def test_sample_top_p_whose_end_lies_below_its_bound():
    """220,000 tokens, each just below the weight at which all of them together would be
    1 - top_p, weigh 4.70 steps and are held as 5: more than 1 - top_p, so the end lies among them
    and not above the bound.  By the weights themselves the first token alone stays; by those held,
    it and the first 10,285 others of 5 2^-44 each.  Either way u, 2^-24 below 1, draws the first."""
    V, p = 220000, 1 - 2.0 ** -24
    bound = math.log(2.0 ** -24 / V) - 0.01
    x = torch.full((2, V), bound - 0.003)
    x[0, 0] = x[1, 0] = 0.0
    step = math.exp(float(x[0, 1])) * 2.0 ** 44
    assert 4.5 < step < 2.0 ** 20 / V                  # rounds upwards, past the share of each
    x[1] += 8.0
    _sample_case(x, torch.full((2,), p), top_p=p)
