"""CPU tests of cr_append_kv and cr_attend at the limits of what a launch can
hold (every call here returns before anything is enqueued)."""
import pytest

from paper_2609_35139_amd import binding as B


def _batch(n_seqs, H, d, offsets=None, L=1, bs=16, max_blocks=256, n_blocks=300):
    lay, sB = B.paged_layout(L, H, d, n_blocks, bs, B.CR_DTYPE_BF16)
    q, keep = B.sequences_struct(n_seqs, 0x7000, 0x8000, max_blocks, bs, n_blocks, sB, offsets)
    q.keep = keep
    return lay, q


def _attend(lay, q, heads, shared=0):
    o = B.cr_attend_options()
    o.shared_len = shared
    rows = [B.cr_rows(at, heads * lay.head_dim, lay.head_dim) for at in (0x100000, 0x500000)]
    with pytest.raises(B.CrError) as e:
        B.cr_attend(0x10000, lay, 0, q, *rows, heads, o, 0x400000, 1 << 60)
    return e.value.name


def _sizes(lay, q, heads, shared=0):
    with pytest.raises(B.CrError) as e:
        B.cr_attend_workspace_bytes(lay, q, heads, shared)
    return e.value.name


def test_attend_with_more_threads_than_a_launch_has():
    """2^32 threads: 131,072 tokens of 256 KV heads, two waves each."""
    lay, q = _batch(1 << 17, 256, 32)
    assert _attend(lay, q, 256) == _sizes(lay, q, 256) == "CR_ERR_DIMS"
    lay, q = _batch((1 << 17) - 1, 256, 32)
    assert B.cr_attend_workspace_bytes(lay, q, 256) == 0      # the most that fit


def test_attend_with_too_many_wide_units():
    """Four waves for each unit of 17 tokens."""
    n = 1 << 16
    lay, q = _batch(n, 256, 32, offsets=range(0, 17 * n + 1, 17))
    assert _attend(lay, q, 256) == _sizes(lay, q, 256) == "CR_ERR_DIMS"
    lay, q = _batch(n - 1, 256, 32, offsets=range(0, 17 * (n - 1) + 1, 17))
    B.cr_attend_workspace_bytes(lay, q, 256)


def test_attend_whose_merge_is_too_large():
    """The pass over shared keys leaves a merge, four waves for each token and
    KV head, where the attention's own launch has two."""
    lay, q = _batch(1 << 16, 256, 32)
    assert _attend(lay, q, 256, 2000) == _sizes(lay, q, 256, 2000) == "CR_ERR_DIMS"
    assert B.cr_attend_workspace_bytes(lay, q, 256) == 0      # no shared keys, no merge


def test_append_with_more_threads_than_a_launch_has():
    """A thread copies eight elements of a value: 2^32 of them."""
    H, d = 1 << 16, 256
    lay, q = _batch(2048, H, d, n_blocks=4, bs=1)
    rows = [B.cr_rows(at, H * d, d) for at in (0x100000, 0x500000)]
    with pytest.raises(B.CrError) as e:
        B.cr_append_kv(0x10000, lay, 0, q, *rows, None, None, 0, None, None)
    assert e.value.name == "CR_ERR_DIMS"


def test_the_serving_kernels_are_among_the_resources_reported():
    """... so that none of them can spill unseen."""
    import os
    from paper_2609_35139_amd import build
    if not os.path.exists(build.RESOURCES):
        pytest.skip("library not built here")
    names = [line.split()[0] for line in open(build.RESOURCES)]
    for element in ("DF16b", "f"):
        for kernel, count in (("append_kernel", 2), ("attend_kernel", 16), ("attend_merge_kernel", 3)):
            assert sum(f"{kernel}I{element}L" in n for n in names) == count, (kernel, element)
