"""Calls of cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample at the
limits of their ranges, on the GPU."""
import math

import numpy as np
import pytest
import torch

from test_gpu_answer import _i32, _layout_cache

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
