"""Calls of cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample at the
limits of their ranges, on the GPU."""
import math

import numpy as np
import pytest
import torch

from serving_helpers import TORCH
from test_gpu_answer import _i32, _layout_cache, _sample_case

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35139_amd import binding
    binding.load()


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
