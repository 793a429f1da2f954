"""cr_append_kv and cr_attend on the GPU against their definitions in 64 bits
(tests/serving_helpers.py), with bounds derived there from the roundings."""
import math

import numpy as np
import pytest
import torch

from serving_helpers import TORCH, Batch, append_oracle, assert_within, attend_oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35139_amd import binding
    binding.load()


# ------------------------------------------------------------------- append
APPEND = {
    "decode": dict(dtype="bf16", heads=16, kv_heads=2, d=128, bs=16, q=[1] * 5, lens=[1, 16, 17, 250, 33]),
    "ragged": dict(dtype="bf16", heads=6, kv_heads=3, d=64, bs=8, q=[0, 5, 1, 40], lens=[9, 5, 30, 41]),
    "f32": dict(dtype="f32", heads=4, kv_heads=4, d=96, bs=1, q=[3, 0, 2], lens=[3, 0, 9]),
    "wide": dict(dtype="bf16", heads=2, kv_heads=1, d=256, bs=1024, q=[33], lens=[1100]),
    "narrow": dict(dtype="f32", heads=5, kv_heads=1, d=32, bs=4, q=[7, 7], lens=[7, 50]),
    # lengths that leave new tokens without a slot
    "short": dict(dtype="bf16", heads=2, kv_heads=2, d=64, bs=4, q=[5, 2, 1], lens=[3, -2, 0]),
}


@pytest.mark.parametrize("name", APPEND)
@pytest.mark.parametrize("far", [None, (1 << 20) + 7, -9])
def test_append(name, far):
    b = Batch(L=2, seed=len(name), fill=7.5, **APPEND[name])
    cache, seqs, q, k, v = b.cuda()
    pos = None
    if far is not None:
        pos = [far + 3 * i for i in range(b.N)]
    got = cache.append(1, seqs, k, v, q=q, rope=dict(theta=1e6, scale=1.25),
                       positions=None if pos is None else torch.tensor(pos, dtype=torch.int32).cuda())
    pool, qo, ep, eq = append_oracle(b, 1, scale=1.25, positions=pos)
    assert_within(cache.pool, pool, ep, "cache")        # what no token was appended to: exactly
    assert_within(got, qo, eq, "queries")


def test_append_copies_without_rope_and_in_place():
    b = Batch(L=1, seed=4, **APPEND["ragged"])
    cache, seqs, q, k, v = b.cuda()
    k[0, 0, 0] = float("nan")
    b.kh[0, 0, 0] = float("nan")
    out = cache.append(0, seqs, k, v, q=q)
    pool, _, ep, _ = append_oracle(b, 0, rotate=False)
    assert_within(cache.pool, pool, ep * 0, "cache")
    assert torch.equal(out, q)
    cache.append(0, seqs, k, v)                          # no queries
    ref = cache.append(0, seqs, k, v, q=q, rope=dict(theta=1e4))
    same = q.clone()
    assert cache.append(0, seqs, k, v, q=same, q_out=same, rope=dict(theta=1e4)) is same
    assert torch.equal(same, ref)


@pytest.mark.parametrize("dtype,heads,kv_heads,d", [("bf16", 14, 3, 128), ("f32", 5, 1, 256),
                                                    ("bf16", 24, 4, 96)])
def test_append_of_many_tokens(dtype, heads, kv_heads, d):
    """Enough tokens for several heads to a thread, heads that do not divide
    evenly among them; queries rotated where they lie."""
    b = Batch(dtype, heads, kv_heads, d, 16, [700, 0, 1, 41], [900, 5, 300, 41], seed=19)
    cache, seqs, q, k, v = b.cuda()
    pool, qo, ep, eq = append_oracle(b, 0)
    got = cache.append(0, seqs, k, v, q=q, q_out=q, rope=dict(theta=1e6))
    assert got.data_ptr() == q.data_ptr()
    assert_within(cache.pool, pool, ep, "cache")
    assert_within(got, qo, eq, "queries")


def test_append_frequency_table_and_many_sequences():
    """300 sequences of zero to two tokens (more than one launch's table), the
    model's own frequencies."""
    q = [i % 3 for i in range(300)]
    b = Batch("bf16", 4, 2, 64, 4, q, [n + i % 7 for i, n in enumerate(q)], seed=9)
    cache, seqs, qh, k, v = b.cuda()
    f = [1e4 ** (-i / 32) / (1 + i % 2) for i in range(32)]
    got = cache.append(0, seqs, k, v, q=qh, rope=dict(inv_freq=f))
    pos = torch.tensor([j for _, j in b.slots()], dtype=torch.float64)
    ang = pos[:, None, None] * torch.tensor(f, dtype=torch.float32).double()
    u, w = b.qh[..., :32].double(), b.qh[..., 32:].double()
    ref = torch.cat([u * ang.cos() - w * ang.sin(), w * ang.cos() + u * ang.sin()], -1)
    size = torch.cat([u.abs() + w.abs()] * 2, -1)
    assert_within(got, ref, 2.0 ** -20 * size + 2.0 ** -8 * ref.abs(), "queries")


def test_append_drops_tokens_of_no_block():
    b = Batch("bf16", 2, 2, 64, 4, [6, 6], [10, 12], seed=5, fill=7.5)
    b.table[0, 1], b.table[1, 2] = -1, b.n_blocks       # slots 4-7, slots 8-11
    cache, seqs, q, k, v = b.cuda()
    got = cache.append(0, seqs, k, v, q=q, rope=dict(theta=1e6))
    pool, qo, ep, eq = append_oracle(b, 0)
    assert_within(cache.pool, pool, ep, "cache")
    assert_within(got, qo, eq, "queries")


# ------------------------------------------------------------------- attend
def _check(b, layer=0, shared=0, what="", **opt):
    """attend against the oracle, twice to the same bits."""
    cache, seqs, q, _, _ = b.cuda()
    dev = {k: torch.tensor(v, dtype=torch.int32).cuda() if k in ("lo", "hi") else v
           for k, v in opt.items()}
    lse = torch.empty(b.N, b.heads, device="cuda")
    out = cache.attend(layer, seqs, q, lse=lse, shared_len=shared, **dev)
    again = cache.attend(layer, seqs, q, shared_len=shared, **dev)
    ref, rl, tol, ltol = attend_oracle(b, layer, **opt)
    assert_within(out, ref, tol, what + "out")
    assert_within(lse, rl, ltol, what + "lse")
    assert torch.equal(out.view(torch.int16 if b.dtype == "bf16" else torch.int32),
                       again.view(torch.int16 if b.dtype == "bf16" else torch.int32))
    return out


ATTEND = {
    "decode": dict(dtype="bf16", heads=16, kv_heads=2, d=128, bs=16, q=[1] * 8,
                   lens=[1, 2, 63, 64, 65, 300, 1000, 17]),
    "decode-f32": dict(dtype="f32", heads=4, kv_heads=2, d=128, bs=16, q=[1] * 4, lens=[1, 31, 129, 700]),
    "ragged": dict(dtype="bf16", heads=12, kv_heads=4, d=64, bs=8, q=[0, 1, 17, 130, 5],
                   lens=[4, 200, 17, 300, 700]),
    "ragged-f32": dict(dtype="f32", heads=6, kv_heads=2, d=64, bs=4, q=[3, 0, 41], lens=[3, 5, 150]),
    "one-token": dict(dtype="bf16", heads=2, kv_heads=2, d=64, bs=1, q=[1], lens=[1]),
    "many-heads": dict(dtype="bf16", heads=40, kv_heads=1, d=64, bs=16, q=[1, 4], lens=[90, 260]),
    "group-of-7": dict(dtype="bf16", heads=28, kv_heads=4, d=128, bs=16, q=[1, 9, 1], lens=[70, 80, 500]),
    "prompt": dict(dtype="bf16", heads=4, kv_heads=2, d=128, bs=64, q=[333], lens=[333]),
    "long": dict(dtype="bf16", heads=2, kv_heads=1, d=128, bs=16, q=[1], lens=[20001]),
    "long-pages-of-1": dict(dtype="bf16", heads=2, kv_heads=1, d=64, bs=1, q=[2], lens=[2500]),
    "pages-of-1024": dict(dtype="bf16", heads=2, kv_heads=1, d=64, bs=1024, q=[1, 1], lens=[1025, 3000]),
    "d32": dict(dtype="bf16", heads=4, kv_heads=2, d=32, bs=16, q=[1, 20], lens=[100, 77]),
    "d96": dict(dtype="bf16", heads=4, kv_heads=2, d=96, bs=16, q=[1, 20], lens=[100, 277]),
    "d160": dict(dtype="bf16", heads=4, kv_heads=2, d=160, bs=16, q=[1, 20], lens=[100, 77]),
    "d224-f32": dict(dtype="f32", heads=4, kv_heads=2, d=224, bs=16, q=[1, 20], lens=[100, 77]),
    "d192-f32": dict(dtype="f32", heads=2, kv_heads=2, d=192, bs=2, q=[70], lens=[90]),
    "d256": dict(dtype="bf16", heads=4, kv_heads=1, d=256, bs=16, q=[1, 50], lens=[400, 77]),
    "d256-f32": dict(dtype="f32", heads=4, kv_heads=1, d=256, bs=16, q=[1, 30], lens=[300, 77]),
    # lengths that leave queries without a key of their own
    "short": dict(dtype="bf16", heads=4, kv_heads=2, d=64, bs=4, q=[5, 2, 1, 3], lens=[3, -2, 0, 40]),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attend_causal(name):
    # rows of the cache in no sequence's slots hold NaN: they are never seen
    _check(Batch(L=2, seed=len(name), fill=float("nan"), table_slack=1, **ATTEND[name]), layer=1)


@pytest.mark.parametrize("name", ["decode", "ragged", "ragged-f32", "group-of-7", "d96", "d256-f32", "short"])
@pytest.mark.parametrize("kind", ["capped", "bias", "capped-bias-documents", "windows", "all"])
def test_attend_options(name, kind):
    b = Batch(seed=3 + len(kind), **ATTEND[name])
    rng = np.random.default_rng(7)
    p = np.array([j for _, j in b.slots()])
    n = np.repeat(np.maximum(b.lens, 0), b.q)
    slopes = [2.0 ** (-8.0 * (h + 1) / b.heads) for h in range(b.heads)]
    opt = {}
    if "capped" in kind:
        opt["softcap"] = 5.0
    if "bias" in kind:
        opt["slopes"] = slopes
    if "documents" in kind:                       # every third query sees nothing
        opt["lo"] = rng.integers(-3, np.maximum(p, 0) + 1)
        opt["hi"] = np.where(np.arange(b.N) % 3 == 0, opt["lo"], p + 1)
    if kind == "windows":                         # the 20 keys before, none of the later ones
        opt["lo"] = p - 20
    if kind == "all":                             # hi beyond the length, a scale of its own
        opt["hi"] = n + 1000
        opt["scale"] = 0.3
    _check(b, **opt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", range(32, 257, 32))
def test_every_head_dim(dtype, d):
    """One token each and questions, split and whole."""
    for q, lens in (([1] * 3, [40, 500, 129]), ([1, 40, 9], [30, 900, 200])):
        b = Batch(dtype, 4, 2, d, 16, q, lens, seed=23)
        _check(b)
        p = np.array([j for _, j in b.slots()])
        _check(b, softcap=10.0, slopes=[0.02, 0.0, 0.3, 0.01], lo=p - 70, hi=p + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_hidden_keys_do_not_matter(dtype):
    """Infinities and NaN in keys that some rows of a tile see and others do
    not: a padded batch, documents of another query."""
    b = Batch(dtype, 4, 2, 64, 8, [40, 3], [60, 3], seed=21)
    slot = {(s, j): t for t, (s, j) in enumerate(b.slots())}
    hidden = {}
    for j, kv, x in [(33, 1, float("inf")), (45, 1, float("nan")), (50, 1, -float("inf")),
                     (52, 0, float("nan")), (58, 0, float("inf"))]:
        at = b.row(0, j)
        b.pool[0, kv, at[0], at[1], 1, 5] = x
        hidden[j] = x
    out = _check(b)
    first = slot[(0, 33)]
    assert torch.isfinite(out[:first]).all()      # rows before the first odd value: finite
    assert torch.isfinite(out[:, :2]).all()       # the other KV head never
    assert torch.isnan(out[slot[(0, 46)], 2:, 5]).all() and torch.isinf(out[slot[(0, 40)], 2:, 5]).all()
    lo = np.zeros(b.N, int)
    lo[:40] = 59
    hi = np.full(b.N, 60)
    hi[5] = 0
    out = _check(b, lo=lo, hi=hi)                 # every query sees one key, one sees none
    assert torch.isfinite(out).all() and (out[5] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q", [1, 40])
def test_extreme_intervals(dtype, q):
    """Limits at the ends of their type, in tiles that other rows see."""
    b = Batch(dtype, 4, 2, 64, 16, [q] * 3, [400, 90, 700], seed=25)
    least, most = -2 ** 31, 2 ** 31 - 1
    t = np.arange(b.N)
    p = np.array([j for _, j in b.slots()])
    lo = np.choose(t % 5, [least, 0, most, p, -7])
    hi = np.choose(t % 4, [most, least, p + 1, p + 9])
    _check(b, lo=lo, hi=hi)


def test_factors_beyond_their_type():
    """Scales and slopes whose product with log2 e is no fp32 number: scores of
    zero and keys at no distance stay what they are."""
    b = Batch("bf16", 4, 2, 64, 16, [1, 1], [1, 200], seed=27)
    cache, seqs, q, _, _ = b.cuda()
    zero = torch.zeros_like(q.contiguous())
    ref, _, tol, _ = attend_oracle(b, 0, q=zero.cpu())
    for opt in (dict(scale=3.3e38), dict(softcap=3.3e38), dict(softcap=1e-40)):
        assert_within(cache.attend(0, seqs, zero, **opt), ref, tol, str(opt))
    out = cache.attend(0, seqs, zero, slopes=[3.3e38] * 4)      # itself alone
    own = torch.stack([b.pool[0, 1, r[0], r[1]] for r in (b.row(0, 0), b.row(1, 199))])
    assert torch.equal(out.cpu(), own.repeat_interleave(2, 1))


def test_blocks_that_are_none_are_not_seen():
    b = Batch("bf16", 4, 2, 64, 4, [1, 30], [200, 90], seed=22)
    b.table[0, 3], b.table[0, 20], b.table[1, 2], b.table[1, 22] = -1, b.n_blocks, 1 << 30, -(1 << 31)
    _check(b)
    b.table[:] = -1
    out = _check(b)
    assert (out == 0).all()


def test_length_beyond_the_table_counts_as_the_table():
    b = Batch("bf16", 4, 2, 64, 4, [1, 2], [41, 16], seed=23)
    cache, _, q, _, _ = b.cuda()
    lens = torch.tensor([1 << 30, 16], dtype=torch.int32).cuda()
    seqs = cache.sequences(b.table.cuda(), lens, b.off)
    b.lens = [44, 16]
    out = cache.attend(0, seqs, q)
    ref, _, tol, _ = attend_oracle(b, 0)
    assert_within(out, ref, tol, "out")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("shared,q,lens", [
    (64, [1] * 6, [64, 65, 100, 2, 700, 128]),        # a sequence that ends inside the prefix
    (1100, [1, 3, 0, 20], [1101, 1180, 1100, 1500]),
    (999, [2, 2], [1200, 1003]),                      # ends inside a page
])
def test_shared_prefix(dtype, d, shared, q, lens):
    b = Batch(dtype, 8, 2, d, 16, q, lens, seed=31, shared=-(-shared // 16) * 16)
    plain = _check(b)
    out = _check(b, shared=shared, what="shared ")
    assert (out.float() - plain.float()).abs().max() < (2.0 ** -6 if dtype == "bf16" else 1e-5)
    p = np.array([j for _, j in b.slots()])
    _check(b, shared=shared, lo=p - 300, hi=np.where(p % 4 == 1, 0, p + 1), softcap=8.0,
           slopes=[0.01 * h for h in range(8)])


def _launched(call):
    """(result, names of the launches) of a call."""
    from paper_2609_35139_amd import binding as B
    B.cr_profile_enable(64)
    try:
        out = call()
        return out, {r["name"] for r in B.cr_profile_read()}
    finally:
        B.cr_profile_enable(0)


READ_ONCE = {
    # tokens of many sequences; some end inside the prefix, some see nothing
    "tokens": dict(dtype="bf16", heads=16, kv_heads=8, d=128, q=[1] * 120, shared=1000,
                   more=lambda s: [37, -400, 300, 1, -1000, 129][s % 6]),
    # more sequences than travel with a launch, rows that fill no unit; with the
    # shorter prefix the pass would cost more than it saves
    "questions": dict(dtype="bf16", heads=24, kv_heads=4, d=128, q=[3, 4, 0, 5] * 44, shared=2201,
                      more=lambda s: 7 + s % 90),
    "questions-short": dict(dtype="bf16", heads=24, kv_heads=4, d=128, q=[3, 4, 0, 5] * 44,
                            shared=1001, more=lambda s: 7 + s % 90, once=False),
    "f32": dict(dtype="f32", heads=8, kv_heads=8, d=64, q=[1] * 100, shared=900,
                more=lambda s: s % 80),
    "d256": dict(dtype="bf16", heads=8, kv_heads=8, d=256, q=[1] * 70, shared=600,
                 more=lambda s: 3 * s),
    # no unit is split: as many as fill the chip
    "many": dict(dtype="bf16", heads=8, kv_heads=8, d=64, q=[1] * 1040, shared=700,
                 more=lambda s: 1 + s % 20),
    # 512 parts of the prefix and one more, for a few rows
    "far": dict(dtype="bf16", heads=1, kv_heads=1, d=64, q=[1] * 16, shared=131072,
                more=lambda s: 5 * s),
    # 56 parts of the prefix and 14 more, for many rows
    "wide-group": dict(dtype="bf16", heads=16, kv_heads=1, d=128, q=[1] * 70, shared=14336,
                       more=lambda s: 1800 - s),
}


@pytest.mark.parametrize("name", READ_ONCE)
def test_shared_prefix_read_once(name):
    """Batches for which the pass over the shared keys pays (but one), and
    without it, against the oracle."""
    c = dict(READ_ONCE[name])
    shared, more, once = c.pop("shared"), c.pop("more"), c.pop("once", True)
    lens = [shared + more(s) for s in range(len(c["q"]))]
    b = Batch(lens=lens, bs=16, seed=33, shared=-(-shared // 16) * 16, **c)
    cache, seqs, q, _, _ = b.cuda()
    lse = torch.empty(b.N, b.heads, device="cuda")
    out, names = _launched(lambda: cache.attend(0, seqs, q, lse=lse, shared_len=shared))
    assert ("attend_shared" in names) == once
    plain, names = _launched(lambda: cache.attend(0, seqs, q))
    assert "attend_shared" not in names
    assert torch.equal(out, cache.attend(0, seqs, q, shared_len=shared))
    tell = range(b.N) if name in ("tokens", "f32", "d256", "far") else range(0, b.N, 7)
    ref, rl, tol, ltol = attend_oracle(b, 0, tokens=tell)
    for what, x in (("shared", out), ("plain", plain)):
        assert_within(x[list(tell)], ref[list(tell)], tol[list(tell)], what)
    assert_within(lse[list(tell)], rl[list(tell)], ltol[list(tell)], "lse")


def test_shared_prefix_masked_and_replayed():
    """The pass over shared keys under windows, a cap and distance slopes, in a
    captured graph that is replayed while the queries change."""
    shared, n = 1000, 120
    b = Batch("bf16", 16, 8, 128, 16, [1] * n, [shared + s % 50 for s in range(n)], seed=35,
              shared=1008)
    cache, seqs, q, _, _ = b.cuda()
    p = np.array([j for _, j in b.slots()])
    lo, hi = p - 300 - 7 * np.arange(n), np.where(p % 4 == 1, 0, p + 1)
    opt = dict(softcap=8.0, slopes=[0.01 * h for h in range(16)])
    dev = dict(lo=torch.tensor(lo, dtype=torch.int32).cuda(),
               hi=torch.tensor(hi, dtype=torch.int32).cuda(), shared_len=shared, **opt)
    q = q.contiguous()
    first, names = _launched(lambda: cache.attend(0, seqs, q, **dev))
    assert "attend_shared" in names
    ref, _, tol, _ = attend_oracle(b, 0, lo=lo, hi=hi, **opt)
    assert_within(first, ref, tol, "masked")
    ws, out = cache.workspace(seqs, 16, shared), torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(0, seqs, q, out=out, workspace=ws, **dev)
    for i in range(4):
        q.mul_(0.9)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, cache.attend(0, seqs, q, **dev)), i


@pytest.mark.parametrize("name", ["plan-of-200", "tokens-unsplit", "questions-unsplit", "even",
                                  "uneven", "even-tokens", "uneven-tokens", "short-table"])
def test_how_a_batch_is_split(name):
    """Batches whose units are planned beyond one wave's worth, are too many to
    split, or are split or left whole by the device's rule."""
    c = {
        "plan-of-200": dict(heads=2, kv_heads=1, d=64, q=[s % 21 for s in range(200)],
                            lens=[21 + (37 * s) % 300 for s in range(200)]),
        "tokens-unsplit": dict(heads=8, kv_heads=8, d=64, q=[1] * 1030,
                               lens=[1 + (13 * s) % 280 for s in range(1030)]),
        "questions-unsplit": dict(heads=16, kv_heads=16, d=64, q=[17] * 33,
                                  lens=[17 + 11 * s for s in range(33)]),
        "even": dict(heads=16, kv_heads=4, d=128, q=[32] * 20, lens=[332] * 20),
        "uneven": dict(heads=16, kv_heads=4, d=128, q=[32, 9, 17], lens=[4000, 32, 600]),
        "even-tokens": dict(heads=8, kv_heads=8, d=64, q=[1] * 64, lens=[700 - s for s in range(64)]),
        "uneven-tokens": dict(heads=8, kv_heads=8, d=64, q=[1] * 64, lens=[3000] + [100] * 63),
        "short-table": dict(heads=4, kv_heads=2, d=64, q=[1] * 3, lens=[500, 512, 1]),
    }[name]
    _check(Batch("bf16", bs=16, seed=37, **c))


def test_sequences_of_another_cache():
    b = Batch("bf16", 4, 2, 64, 16, [1], [30], seed=41)
    cache, seqs, q, k, v = b.cuda()
    other = type(cache)(cache.pool[:, :, :1])
    for call in (lambda: other.attend(0, seqs, q), lambda: other.append(0, seqs, k, v),
                 lambda: other.workspace(seqs, 4)):
        with pytest.raises(ValueError):
            call()


def test_workspace_that_is_no_memory_of_its_size():
    b = Batch("bf16", 4, 2, 64, 16, [1], [900], seed=43)
    cache, seqs, q, _, _ = b.cuda()
    need = cache.workspace(seqs, 4).numel()
    for ws in (torch.empty(1, dtype=torch.uint8, device="cuda").expand(need),
               torch.empty(need, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            cache.attend(0, seqs, q, workspace=ws)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own."""
    b = Batch("bf16", 8, 2, 128, 16, [1] * 6, [3000, 40, 900, 2500, 1, 700], seed=39)
    cache, seqs, q, _, _ = b.cuda()
    q = q.contiguous()
    want = cache.attend(0, seqs, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [cache.workspace(seqs, 8) for _ in streams]
    outs = [torch.empty(20, *q.shape, dtype=q.dtype, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(20):
        for s, w, o in zip(streams, ws, outs):
            cache.attend(0, seqs, q, out=o[i], workspace=w, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(x, want) for x in o)


def test_pool_of_other_strides_and_strided_rows():
    """Block-major pool with K and V and layers inside a block; queries and
    results with strides of their own; only the result's rows are written."""
    b = Batch("bf16", 4, 2, 64, 8, [9, 1], [50, 30], L=3, seed=41)
    from paper_2609_35139_amd.serving import PagedCache
    pool = torch.empty(b.n_blocks, 3, 2, 2, 8, 64 + 8, dtype=torch.bfloat16, device="cuda")
    view = pool[..., :64].permute(1, 2, 0, 4, 3, 5)     # [L][2][n_blocks][bs][H][d]
    view.copy_(b.pool.cuda())
    cache = PagedCache(view)
    seqs = cache.sequences(b.table.cuda(), torch.tensor(b.lens, dtype=torch.int32).cuda(), b.off)
    out = torch.full((4, b.N + 2, 80), 3.0, dtype=torch.bfloat16, device="cuda")
    o = out[:, 1:-1, 8:72].permute(1, 0, 2)
    q = b.qh.permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2)
    cache.attend(2, seqs, q, out=o)
    ref, _, tol, _ = attend_oracle(b, 2)
    assert_within(o, ref, tol, "out")
    o.fill_(3.0)
    assert (out == 3.0).all()
    k, v = b.kh.cuda().expand(-1, 2, -1), b.vh[:, :1].cuda().expand(-1, 2, -1)   # one value for both heads
    b.vh = b.vh[:, :1].expand(-1, 2, -1)
    cache.append(0, seqs, k, v, rope=dict(theta=1e6))
    p, _, ep, _ = append_oracle(b, 0)
    assert_within(view, p, ep, "cache")


def test_offsets_past_32_bits():
    """Pages beyond 2^32 elements of a pool of 9.7 GB."""
    from paper_2609_35139_amd.serving import PagedCache
    b = Batch("bf16", 4, 2, 128, 16, [1, 5], [40, 90], seed=43)
    far = 600_000
    pool = torch.empty(1, 2, far + b.n_blocks, 16, 2, 128, dtype=torch.bfloat16, device="cuda")
    pool[:, :, far:] = b.pool.cuda()
    cache = PagedCache(pool)
    table = torch.where(b.table >= 0, b.table + far, b.table).cuda()
    seqs = cache.sequences(table, torch.tensor(b.lens, dtype=torch.int32).cuda(), b.off)
    q = cache.append(0, seqs, b.kh.cuda(), b.vh.cuda(), q=b.qh.cuda(), rope=dict(theta=1e6))
    p, qo, ep, eq = append_oracle(b, 0)
    assert_within(pool[:, :, far:], p, ep, "cache")
    assert_within(q, qo, eq, "queries")
    out = cache.attend(0, seqs, q)
    ref, _, tol, _ = attend_oracle(b, 0, pool=pool[:, :, far:].cpu(), q=q.cpu())
    assert_within(out, ref, tol, "out")


# ---------------------------------------------------------------- in a program
def test_decode_steps_in_a_captured_graph_on_another_stream():
    """A captured step (append, attend, two layers) replayed while lengths,
    tables and inputs move on, against the same step run eagerly and against
    the definition; two graphs share one workspace, in turn."""
    from paper_2609_35139_amd.serving import PagedCache
    b = Batch("bf16", 8, 2, 64, 4, [1] * 3, [90, 700, 5], L=2, seed=51, spare=40)
    table = torch.full((3, 190), -1, dtype=torch.int32)
    table[:, :b.table.shape[1]] = b.table
    free = [i for i in range(b.n_blocks) if i not in set(b.table.flatten().tolist())]
    for s, n in enumerate(b.lens):                       # room for the steps to come
        have = -(-n // 4)
        table[s, have:have + 4] = torch.tensor([free.pop() for _ in range(4)])
    b.table = table
    side = torch.cuda.Stream()
    dt, rope = torch.bfloat16, dict(theta=1e6)

    def world():
        cache = PagedCache(b.pool.cuda())
        lens = torch.tensor([n - 1 for n in b.lens], dtype=torch.int32).cuda()
        new = torch.zeros(2, 3, 12, 64, dtype=dt, device="cuda")
        return cache, lens, cache.sequences(table.cuda(), lens), new, torch.zeros(2, 3, 8, 64, dtype=dt, device="cuda")

    def step(w, ws, stream):
        cache, lens, seqs, new, out = w
        for layer in range(2):
            q, k, v = new[layer, :, :8], new[layer, :, 8:10], new[layer, :, 10:]
            q = cache.append(layer, seqs, k, v, q=q, rope=rope, stream=stream)
            cache.attend(layer, seqs, q, out=out[layer], workspace=ws, stream=stream)

    eager, a = world(), world()
    ws = a[0].workspace(a[2], 8)
    side.wait_stream(torch.cuda.current_stream())
    a[1].add_(1)
    step(a, ws, side)                                    # warm-up, over slots written again below
    side.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(a, ws, side)
        graphs.append(g)
    a[1].sub_(1)
    gen = torch.Generator().manual_seed(5)
    for i in range(5):
        x = torch.randn(2, 3, 12, 64, generator=gen).to(dt)
        for w in (eager, a):
            w[1].add_(1)
            w[3].copy_(x)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(eager, None, None)
        assert torch.equal(a[4], eager[4]) and torch.equal(a[0].pool, eager[0].pool)
        b.lens = eager[1].tolist()
        q = eager[0].append(1, eager[2], x[1, :, 8:10].cuda(), x[1, :, 10:].cuda(), q=x[1, :, :8].cuda(), rope=rope)
        ref, _, tol, _ = attend_oracle(b, 1, pool=eager[0].pool.cpu(), q=q.cpu())
        assert_within(a[4][1], ref, tol, f"step {i}")


def test_repaired_cache_is_answered_over():
    """Repair into pages with the keys placed, append a question, attend with
    the documents shared by two questions: the whole path of a request."""
    import workloads as W
    from helpers import repairer_for, small_workload, to_device
    from paper_2609_35139_amd import binding as B
    from paper_2609_35139_amd.serving import PagedCache
    w = small_workload(((70, 61, 29),), dtype="bf16", L=2, H=2, dh=64, E=128, d_c=64, d_b=128,
                       n_heads=2, d_seg=8, ffn_mult=4)
    inp = W.make_inputs(w)
    rep = repairer_for(w, inp.weights)
    bs, doc = 16, 160
    q = [5, 12]
    b = Batch("bf16", 4, 2, 64, bs, q, [doc + n for n in q], L=2, seed=61, shared=doc)
    cache, seqs, qh, k, v = b.cuda()
    lay, sB = B.paged_layout(2, 2, 64, b.n_blocks, bs, B.CR_DTYPE_BF16)
    kv, emb = to_device(w, inp.kv), to_device(w, inp.token_embeds)
    pages = dict(block_size=bs, n_blocks=b.n_blocks, stride_block=sB, block_table=b.table[0, :doc // bs])
    rep.repair(kv, w.chunk_offsets, w.request_chunks, emb,
               options=B.Options(global_rope=dict(theta=1e6), kv_out=cache.pool.data_ptr(),
                                 layout_out=lay, pages_out=pages))
    before = cache.pool.cpu()
    b.pool = before
    assert not torch.equal(before[:, :, b.table[0, 0]], Batch("bf16", 4, 2, 64, bs, q, b.lens, L=2, seed=61, shared=doc).pool[:, :, b.table[0, 0]])
    for layer in range(2):
        b.pool = cache.pool.cpu()
        qr = cache.append(layer, seqs, k, v, q=qh, rope=dict(theta=1e6))
        pool, qo, ep, eq = append_oracle(b, layer)
        assert_within(cache.pool, pool, ep, "cache")
        out = cache.attend(layer, seqs, qr, shared_len=doc)
        ref, _, tol, _ = attend_oracle(b, layer, pool=cache.pool.cpu(), q=qr.cpu())
        assert_within(out, ref, tol, f"layer {layer}")


def test_profile_names_the_launches():
    from paper_2609_35139_amd import binding as B
    b = Batch(seed=1, **ATTEND["decode"])
    cache, seqs, q, k, v = b.cuda()
    B.cr_profile_enable(16)
    try:
        cache.append(0, seqs, k, v, q=q, rope=dict(theta=1e6))
        cache.attend(0, seqs, q)
        stats = {r["name"]: r["launches"] for r in B.cr_profile_read()}
    finally:
        B.cr_profile_enable(0)
    assert stats["append_kv"] == 1 and stats["attend"] == 1
