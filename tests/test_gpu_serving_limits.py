"""cr_append_kv and cr_attend on the GPU at the limits of their arguments,
against their definitions in 64 bits (tests/serving_helpers.py)."""
import numpy as np
import pytest
import torch

from serving_helpers import HALF, Batch, append_oracle, assert_within, attend_oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35139_amd import binding
    binding.load()


class Outgrown(Batch):
    """A batch whose lengths have grown by `more` past what its table was made
    for: slots count from the true length, and those past the table are none."""

    def __init__(self, *args, more, **kwargs):
        super().__init__(*args, **kwargs)
        self.lens = [min(n + m, 2 ** 31 - 1) for n, m in zip(self.lens, more)]

    def slots(self):
        return [(s, max(n, 0) - nq + i)
                for s, (nq, n) in enumerate(zip(self.q, self.lens)) for i in range(nq)]


# ----------------------------------------------- lengths past the block table
PAST = {
    # the last row, the first one past it, tokens on both sides, all past it
    "tokens": dict(dtype="bf16", heads=4, kv_heads=2, d=64, bs=16, q=[1] * 4, lens=[32, 32, 20, 31],
                   more=[0, 1, 12, 2]),
    "questions": dict(dtype="bf16", heads=4, kv_heads=2, d=64, bs=4, q=[6, 6, 3, 9],
                      lens=[48, 48, 48, 40], more=[3, 0, 3, 12]),
    "f32": dict(dtype="f32", heads=3, kv_heads=1, d=96, bs=1, q=[40, 5, 2], lens=[50, 50, 9],
                more=[7, 50, 2]),
    "far": dict(dtype="bf16", heads=2, kv_heads=2, d=64, bs=16, q=[1, 4, 2], lens=[64, 64, 60],
                more=[1 << 30, 1 << 31, 5]),
}


def _past(name):
    c = dict(PAST[name])
    return Outgrown(c.pop("dtype"), c.pop("heads"), c.pop("kv_heads"), c.pop("d"), c.pop("bs"),
                    c.pop("q"), c.pop("lens"), seed=71 + len(name), **c)


@pytest.mark.parametrize("name", PAST)
def test_append_drops_tokens_past_the_table(name):
    """Such a token leaves every row as it was; the others, and all queries,
    take the positions that the length gives them."""
    b = _past(name)
    cache, seqs, q, k, v = b.cuda()
    got = cache.append(0, seqs, k, v, q=q, rope=dict(theta=1e6))
    pool, qo, ep, eq = append_oracle(b, 0)
    # a position's angle is off by four roundings in 64 bits on either side
    pos = torch.tensor([j for _, j in b.slots()], dtype=torch.float64)[:, None, None]
    half = b.d // 2
    size = (b.qh[..., :half].double().abs() + b.qh[..., half:].double().abs()).repeat(1, 1, 2)
    assert_within(cache.pool, pool, ep, "cache")        # rows of no new token: exactly
    assert_within(got, qo, eq + 2.0 ** -50 * pos.abs() * size, "queries")


def test_append_replayed_past_the_table():
    """A captured append whose lengths outgrow the table while it is replayed."""
    b = Batch("bf16", 4, 2, 64, 4, [1, 1], [6, 3], seed=73, table_slack=0)
    cache, _, q, k, v = b.cuda()
    lens = torch.tensor(b.lens, dtype=torch.int32).cuda()
    seqs = cache.sequences(b.table.cuda(), lens)
    out = torch.empty_like(q)
    step = lambda: cache.append(0, seqs, k, v, q=q, q_out=out, rope=dict(theta=1e4))
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    want = Outgrown("bf16", 4, 2, 64, 4, [1, 1], [6, 3], seed=73, more=[0, 0])
    for i in range(6):
        want.lens = [6 + i, 3 + i]
        want.pool = cache.pool.cpu()
        g.replay()
        torch.cuda.synchronize()
        pool, qo, ep, eq = append_oracle(want, 0, theta=1e4)
        assert_within(cache.pool, pool, ep, f"cache {i}")
        assert_within(out, qo, eq, f"queries {i}")
        lens.add_(1)


# (a bias of a billion positions would leave no score its bits)
@pytest.mark.parametrize("name,bias", [(n, False) for n in PAST] +
                         [(n, True) for n in PAST if n != "far"])
def test_attend_past_the_table(name, bias):
    """Queries keep the slots that the length gives them: those in the table
    see up to their own key, those past it everything that the table holds."""
    b = _past(name)
    opt = dict(slopes=[0.05 * (h + 1) for h in range(b.heads)]) if bias else {}
    cache, seqs, q, _, _ = b.cuda()
    lse = torch.empty(b.N, b.heads, device="cuda")
    out = cache.attend(0, seqs, q, lse=lse, **opt)
    ref, rl, tol, ltol = attend_oracle(b, 0, **opt)
    assert_within(out, ref, tol, "out")
    assert_within(lse, rl, ltol, "lse")


@pytest.mark.parametrize("q", [[1] * 120, [5, 9, 0, 7] * 30])
def test_shared_prefix_past_the_table(q):
    """The same with the documents read once, and with limits of the caller's."""
    from paper_2609_35139_amd import binding as B
    lens = [3000 + 20 + s % 40 for s in range(len(q))]
    b = Outgrown("bf16", 16, 8, 64, 16, q, lens, seed=79, shared=3008,
                 more=[s % 3 * 30 for s in range(len(q))])
    cache, seqs, qh, _, _ = b.cuda()
    B.cr_profile_enable(8)
    try:
        out = cache.attend(0, seqs, qh, shared_len=3000)
        assert "attend_shared" in {r["name"] for r in B.cr_profile_read()}
    finally:
        B.cr_profile_enable(0)
    tell = list(range(0, b.N, 5))
    ref, _, tol, _ = attend_oracle(b, 0, tokens=tell)
    assert_within(out[tell], ref[tell], tol[tell], "shared")
    p = np.array([j for _, j in b.slots()])
    lo, hi = p - 90, p + 1
    out = cache.attend(0, seqs, qh, shared_len=3000, lo=torch.tensor(lo, dtype=torch.int32).cuda(),
                       hi=torch.tensor(hi, dtype=torch.int32).cuda())
    ref, _, tol, _ = attend_oracle(b, 0, lo=lo, hi=hi, tokens=tell)
    assert_within(out[tell], ref[tell], tol[tell], "windows")


# ------------------------------------------------------------------ score caps
def _capped(b, cap):
    """(out, lse, bounds) of causal attention with capped scores, in 64 bits.
    A cap leaves its score's error no larger, and adds one that is relative to
    the capped score, whatever the cap: 2^-20."""
    out = torch.zeros(b.N, b.heads, b.d, dtype=torch.float64)
    lse = torch.zeros(b.N, b.heads, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    half = HALF[b.dtype]
    pool, q = b.pool[0].double(), b.qh.double()
    for t, (s, p) in enumerate(b.slots()):
        at = torch.tensor([b.row(s, j) for j in range(p + 1)])
        for h in range(b.heads):
            k, v = (pool[c, at[:, 0], at[:, 1], h * b.kv_heads // b.heads] for c in (0, 1))
            x = (k @ q[t, h]) / b.d ** 0.5
            e = (k.abs() @ q[t, h].abs()).max() / b.d ** 0.5 * (b.d + 8) * 2.0 ** -24
            x = cap * torch.tanh(x / cap)
            e = float(e + 2.0 ** -20 * x.abs().max() + 2.0 ** -21 * (1 + x.abs().max()))
            w = torch.softmax(x, 0)
            out[t, h], lse[t, h] = w @ v, torch.logsumexp(x, 0)
            # (the terms of serving_helpers.attend_oracle)
            ltol[t, h] = 2 * e + 2.0 ** -16 + (half if b.dtype == "bf16" else 0.0)
            tol[t, h] = ltol[t, h] * (w @ v.abs() + out[t, h].abs()) + half * out[t, h].abs()
    return out, lse, tol, ltol


@pytest.mark.parametrize("cap", [1e-3, 0.7, 6.0, 30.0, 1e3, 1e5, 1e8, 1e30, 3e38])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_caps_of_every_size(dtype, cap):
    """Scores from far below the cap to far above it; a large cap changes
    nothing.  Single tokens, and questions in whole and in masked tiles."""
    for q, lens in (([1] * 3, [300, 70, 1]), ([40, 7], [400, 90])):
        b = Batch(dtype, 4, 2, 64, 16, q, lens, seed=83)
        b.pool[:, 0] *= 3                    # scores of about 3
        cache, seqs, qh, _, _ = b.cuda()
        lse = torch.empty(b.N, b.heads, device="cuda")
        out = cache.attend(0, seqs, qh, softcap=cap, lse=lse)
        ref, rl, tol, ltol = _capped(b, cap)
        assert_within(out, ref, tol, f"out {q}")
        assert_within(lse, rl, ltol, f"lse {q}")


# ----------------------------------------------------------------- roundings
@pytest.mark.parametrize("far", [0, 1 << 20])
def test_append_rounds_cosines_and_sines_once(far):
    """fp32: of a rotated pair's element only the cosine, the sine, two products
    and their difference are rounded to 32 bits."""
    b = Batch("f32", 6, 2, 128, 16, [300, 70], [900, 70], seed=89)
    cache, seqs, q, k, v = b.cuda()
    p = [far + j for _, j in b.slots()]
    got = cache.append(0, seqs, k, v, q=q, rope=dict(theta=1e6, scale=1.25),
                       positions=torch.tensor(p, dtype=torch.int32).cuda())
    p = torch.tensor(p, dtype=torch.float64)[:, None, None]
    ang = p * 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)
    c, s = 1.25 * ang.cos(), 1.25 * ang.sin()

    def rotated(x):
        u, w = x[..., :64].double(), x[..., 64:].double()
        y = torch.cat([c * u - s * w, c * w + s * u], -1)
        size = torch.cat([(c * u).abs() + (s * w).abs(), (c * w).abs() + (s * u).abs()], -1)
        # (the angle in 64 bits: four roundings on either side)
        off = 2.0 ** -50 * p * 1.25 * (u.abs() + w.abs()).repeat(1, 1, 2)
        return y, 2.0 ** -24 * (2 * size + y.abs()) + off

    assert_within(got, *rotated(b.qh), "queries")
    ref, tol = rotated(b.kh)
    at = torch.tensor([b.row(*x) for x in b.slots()])
    assert_within(cache.pool[0, 0, at[:, 0], at[:, 1]], ref, tol, "keys")


@pytest.mark.parametrize("d", range(32, 257, 32))
def test_single_tokens_keep_their_weights(d):
    """bf16, calls of at most 16 rows: no probability is rounded to bf16, so the
    result's own rounding is the only one of that size."""
    for q, lens in (([1] * 5, [3, 17, 900, 64, 2500]), ([2, 1], [31, 333])):
        b = Batch("bf16", 8, 2, d, 16, q, lens, seed=97)
        cache, seqs, qh, _, _ = b.cuda()
        lse = torch.empty(b.N, b.heads, device="cuda")
        out = cache.attend(0, seqs, qh, lse=lse)
        ref, rl, tol, ltol = attend_oracle(b, 0)
        # serving_helpers.attend_oracle's bounds, where a weight's own error is
        # 2^-16 and no more than half a step (2^-8) of bf16 comes on top: taken off
        # here for the weights (a part of their sum and of the output's size),
        # 2^-17 put in for the two bf16 parts of a weight
        assert_within(lse, rl, ltol - HALF["bf16"] + 2.0 ** -17, f"lse {q}")
        half = HALF["bf16"]
        rest = tol - half * ref.abs()                       # (rel)(sum of w |v| + |o|)
        fine = rest * ((ltol - half + 2.0 ** -17) / ltol)[..., None] + half * ref.abs()
        assert_within(out, ref, fine, f"out {q}")


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64)])
@pytest.mark.parametrize("q", [1, 40])
def test_values_that_are_not_finite_where_all_rows_see_them(dtype, d, q):
    """Infinities and NaN in the middle of long sequences, in tiles without a
    mask: the dims that hold them become infinite or NaN, no others."""
    b = Batch(dtype, 4, 2, d, 16, [q] * 3, [700, 300, 1500], seed=101)
    odd = {(0, 133): (3, float("inf")), (0, 400): (d - 1, -float("inf")), (1, 77): (8, float("nan")),
           (1, 78): (9, float("inf")), (1, 79): (9, -float("inf")), (2, 1000): (d // 2, -float("inf")),
           (2, 1001): (d // 2, -float("inf"))}
    for (s, j), (i, x) in odd.items():
        at = b.row(s, j)
        b.pool[0, 1, at[0], at[1], 1, i] = x
    cache, seqs, qh, _, _ = b.cuda()
    out = cache.attend(0, seqs, qh)
    ref, _, tol, _ = attend_oracle(b, 0)
    assert_within(out, ref, tol, "out")


# ------------------------------------------------------- how a batch is cut up
SPLIT = {
    # as many units as fill the chip, or tables that hold few keys: no parts
    "many tokens": (False, dict(heads=8, kv_heads=8, q=[1] * 1030, lens=[1 + 13 * s % 280 for s in range(1030)])),
    "many questions": (False, dict(heads=16, kv_heads=16, q=[17] * 33, lens=[17 + 11 * s for s in range(33)])),
    "short table": (False, dict(heads=4, kv_heads=2, q=[1] * 3, lens=[500, 512, 1])),
    "short questions": (False, dict(heads=8, kv_heads=2, q=[20, 30], lens=[100, 128])),
    # parts, joined by a launch of their own (whole units leave it nothing to do)
    "one token": (True, dict(heads=4, kv_heads=2, q=[1], lens=[4000])),
    "even tokens": (True, dict(heads=8, kv_heads=8, q=[1] * 64, lens=[700 - s for s in range(64)])),
    "uneven tokens": (True, dict(heads=8, kv_heads=8, q=[1] * 64, lens=[3000] + [100] * 63)),
    "questions": (True, dict(heads=16, kv_heads=4, q=[32, 9, 17], lens=[4000, 32, 600])),
}


@pytest.mark.parametrize("name", SPLIT)
def test_which_batches_are_split(name):
    from paper_2609_35139_amd import binding as B
    split, c = SPLIT[name]
    b = Batch("bf16", d=64, bs=16, seed=103, **c)
    cache, seqs, qh, _, _ = b.cuda()
    B.cr_profile_enable(8)
    try:
        out = cache.attend(0, seqs, qh)
        assert ("attend_merge" in {r["name"] for r in B.cr_profile_read()}) == split
    finally:
        B.cr_profile_enable(0)
    tell = list(range(0, b.N, max(1, b.N // 64)))
    ref, _, tol, _ = attend_oracle(b, 0, tokens=tell)
    assert_within(out[tell], ref[tell], tol[tell], name)


@pytest.mark.parametrize("dtype,d,q", [("bf16", 128, [1] * 120), ("bf16", 64, [5, 0, 9, 7] * 30),
                                       ("f32", 64, [1] * 120), ("f32", 128, [3, 0, 9, 4] * 20)])
def test_shared_pass_under_masks(dtype, d, q):
    """The pass over shared keys (a prefix that ends inside a page; sequences
    that end inside it, hold nothing or have no query), causal and under
    windows, a cap and distance slopes."""
    from paper_2609_35139_amd import binding as B
    shared = 3001
    lens = [shared + [40, -1700, 300, 9, -3001, 129, 1][s % 7] for s in range(len(q))]
    b = Batch(dtype, 16, 8, d, 16, q, lens, seed=107, shared=3008)
    cache, seqs, qh, _, _ = b.cuda()
    p = np.array([j for _, j in b.slots()])
    tell = list(range(0, b.N, 6))
    for opt in ({}, dict(lo=p - 500, hi=np.where(p % 4 == 1, 0, p + 1), softcap=8.0,
                         slopes=[0.01 * h for h in range(16)])):
        dev = {k: torch.tensor(v, dtype=torch.int32).cuda() if k in ("lo", "hi") else v
               for k, v in opt.items()}
        B.cr_profile_enable(8)
        try:
            out = cache.attend(0, seqs, qh, shared_len=shared, **dev)
            assert "attend_shared" in {r["name"] for r in B.cr_profile_read()}
        finally:
            B.cr_profile_enable(0)
        ref, _, tol, _ = attend_oracle(b, 0, tokens=tell, **opt)
        assert_within(out[tell], ref[tell], tol[tell], str(sorted(opt)))
